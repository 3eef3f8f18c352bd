// Host side of the entry points of include/qknorm_attn.h: validation, variant choice, launch.
// Included by qknorm_api.cu INSIDE its unnamed namespace, after the helpers it uses (device cache,
// occupancy cache, overlap test, launch_overlapped).
#pragma once

// ---- rotary positions and the cache write ---------------------------------------------------------

int rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double original_len, double low,
                     double high, double* inv_freq, float* mscale) {
  if (!inv_freq || !mscale) return QKNORM_ERR_NULL;
  if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > QKNORM_MAX_HEAD_DIM) return QKNORM_ERR_SHAPE;
  if (!(theta > 1.0) || !isfinite(theta)) return QKNORM_ERR_SHAPE;
  if (scaling < QKNORM_ROPE_PLAIN || scaling > QKNORM_ROPE_BANDS) return QKNORM_ERR_SHAPE;
  if (scaling != QKNORM_ROPE_PLAIN && !(factor >= 1.0 && isfinite(factor))) return QKNORM_ERR_SHAPE;
  const bool by_turns = scaling == QKNORM_ROPE_RAMP || scaling == QKNORM_ROPE_BANDS;
  if (by_turns && !(original_len > 0.0 && isfinite(original_len) && low > 0.0 && high > low && isfinite(high))) return QKNORM_ERR_SHAPE;
  if (scaling == QKNORM_ROPE_BASE && rot_dim == 2) return QKNORM_ERR_SHAPE;  // its exponent divides by rot_dim - 2
  const double pi2 = 6.283185307179586476925;
  const double base = scaling == QKNORM_ROPE_BASE ? theta * pow(factor, (double)rot_dim / (rot_dim - 2)) : theta;
  *mscale = scaling == QKNORM_ROPE_RAMP ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  // pair index (as a real number) that turns `turns` times within original_len
  auto index_of = [&](double turns) { return rot_dim * log(original_len / (turns * pi2)) / (2.0 * log(theta)); };
  double first = 0.0, last = 0.0;
  if (scaling == QKNORM_ROPE_RAMP) {
    first = fmax(floor(index_of(high)), 0.0);
    last = fmin(ceil(index_of(low)), rot_dim - 1.0);
    if (last <= first) last = first + 0.001;
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / rot_dim);
    double keep = 1.0;  // share of the unscaled frequency
    if (scaling == QKNORM_ROPE_LINEAR) keep = 0.0;
    if (scaling == QKNORM_ROPE_RAMP) keep = 1.0 - fmin(fmax((i - first) / (last - first), 0.0), 1.0);
    if (scaling == QKNORM_ROPE_BANDS) keep = fmin(fmax((original_len * f / pi2 - low) / (high - low), 0.0), 1.0);
    if (scaling != QKNORM_ROPE_PLAIN && scaling != QKNORM_ROPE_BASE) f = f * keep + f / factor * (1.0 - keep);
    inv_freq[i] = f;
  }
  return QKNORM_OK;
}

// A rotation of a call; r == nullptr: none.
int check_rotation(const qknorm_rotation* r, int head_dim, RopeParams& R) {
  R.rot_dim = 0;
  R.mscale = 1.0f;
  if (!r || r->rot_dim == 0) return QKNORM_OK;
  if (r->rot_dim < 0 || r->rot_dim % 2 != 0 || r->rot_dim > head_dim) return QKNORM_ERR_SHAPE;
  if (r->interleaved != 0 && r->interleaved != 1) return QKNORM_ERR_SHAPE;
  if (!isfinite(r->mscale)) return QKNORM_ERR_SHAPE;
  if (!r->positions || !r->inv_freq) return QKNORM_ERR_NULL;
  if ((((uintptr_t)r->positions) | ((uintptr_t)r->inv_freq)) & 7u) return QKNORM_ERR_ALIGN;
  R.rot_dim = r->rot_dim;
  R.interleaved = r->interleaved;
  R.mscale = r->mscale;
  R.positions = (const long long*)r->positions;
  R.inv_freq = r->inv_freq;
  R.turns_sign = 0.15915494309189533577;  // 1 / (2 pi)
  return QKNORM_OK;
}

// The same with several axes.
int check_rotation(const qknorm_rotation_axes* r, int head_dim, RopeParams& R, int64_t T) {
  if (r && r->rot_dim != 0) {
    if (r->num_axes < 1 || r->num_axes > QKNORM_MAX_AXES) return QKNORM_ERR_SHAPE;
    if (r->ld_positions < 0 || (r->ld_positions != 0 && r->ld_positions < T)) return QKNORM_ERR_SHAPE;
    R.axis = r->axis;
    R.axes = r->num_axes;
    R.ld_pos = r->ld_positions ? r->ld_positions : T;
    const qknorm_rotation one = {r->positions, r->inv_freq, r->rot_dim, r->interleaved, r->mscale};
    return check_rotation(&one, head_dim, R);
  }
  return check_rotation((const qknorm_rotation*)nullptr, head_dim, R);
}
int check_rotation(const qknorm_rotation* r, int head_dim, RopeParams& R, int64_t) { return check_rotation(r, head_dim, R); }

struct CallRegions {  // buffers of a call: outputs, and everything an output must not touch
  Region out[8], in[16];
  int outs = 0, ins = 0;
  int own[8];            // out[i] may be exactly in[own[i]]
  int pools = -1, num_pools = 2;  // out[pools] and the num_pools - 1 behind it are the sides of a cache, looked at apart from the others
  bool both_pools(int i, int j) const { return pools >= 0 && i >= pools && j >= pools && i < pools + num_pools && j < pools + num_pools; }
};

int log2_or_minus_one(int v) {
  for (int s = 0; s < 31; ++s)
    if (v == (1 << s)) return s;
  return -1;
}

Region flat(const void* p, uintptr_t bytes) { return Region{(uintptr_t)p, 1, bytes, bytes}; }

// Outputs against every input and every other output; an output may be exactly its own input.
int check_regions(const CallRegions& c) {
  for (int i = 0; i < c.outs; ++i) {
    for (int j = 0; j < c.ins; ++j)
      if (may_overlap(c.out[i], c.in[j]) && !(c.own[i] == j && same_region(c.out[i], c.in[j]))) return QKNORM_ERR_ALIAS;
    for (int j = 0; j < c.outs; ++j)
      if (j != i && !c.both_pools(i, j) && may_overlap(c.out[i], c.out[j])) return QKNORM_ERR_ALIAS;
  }
  return QKNORM_OK;
}

// What a rotation reads.
void rotation_regions(const RopeParams& R, CallRegions& c) {
  if (!R.rot_dim) return;
  const uintptr_t bytes = 8 * (uintptr_t)R.T;
  c.in[c.ins++] = R.axis ? Region{(uintptr_t)R.positions, (uintptr_t)R.axes, bytes, 8 * (uintptr_t)R.ld_pos} : flat(R.positions, bytes);
  c.in[c.ins++] = flat(R.inv_freq, 4 * (uintptr_t)R.rot_dim);
  if (R.axis) c.in[c.ins++] = flat(R.axis, (uintptr_t)R.rot_dim / 2);
}

int row_stride(int64_t ld, int32_t width, long long* out) {
  if (ld < 0 || (ld != 0 && ld < width)) return QKNORM_ERR_SHAPE;
  *out = ld ? ld : width;
  return QKNORM_OK;
}

// Where the elements of one side of a paged cache lie: runs of `width` bytes, along up to three axes from the shortest stride to the
// longest.  nested: every stride is at least as long as all that lies inside it, so that no two runs meet.
struct PoolShape {
  uintptr_t base;
  int64_t width;
  int axes;
  int64_t stride[3], n[3];
  bool nested;
};

PoolShape pool_shape(const qknorm_paged_cache& c, void* base, int64_t page, int64_t token, int64_t head) {
  const int64_t eb = c.e4m3 ? 1 : 2;
  PoolShape s = {(uintptr_t)base, c.head_dim * eb, 0, {0, 0, 0}, {0, 0, 0}, true};
  const int64_t stride[3] = {token * eb, head * eb, page * eb}, n[3] = {c.page_size, c.heads, c.num_pages};
  for (int a = 0; a < 3; ++a) {
    if (n[a] <= 1) continue;
    int i = s.axes++;
    for (; i > 0 && s.stride[i - 1] > stride[a]; --i) {
      s.stride[i] = s.stride[i - 1];
      s.n[i] = s.n[i - 1];
    }
    s.stride[i] = stride[a];
    s.n[i] = n[a];
  }
  int64_t inside = s.width;
  for (int i = 0; i < s.axes; ++i) {
    s.nested = s.nested && s.stride[i] >= inside;
    inside += (s.n[i] - 1) * s.stride[i];
  }
  return s;
}

// The side as rows of one pitch: axes without gaps become the row, those that go on evenly its repetitions; what an axis
// beyond them leaves free counts as taken.
Region pool_region(const PoolShape& s) {
  int64_t width = s.width, rows = 1, pitch = 0;
  for (int i = 0; i < s.axes; ++i) {
    if (rows == 1 && s.stride[i] == width) {
      width *= s.n[i];
    } else if (rows == 1 || s.stride[i] == rows * pitch) {
      pitch = rows == 1 ? s.stride[i] : pitch;
      rows *= s.n[i];
    } else {
      width += (rows - 1) * pitch;
      pitch = s.stride[i];
      rows = s.n[i];
    }
  }
  if (!s.nested) {
    width = s.width;
    for (int i = 0; i < s.axes; ++i) width += (s.n[i] - 1) * s.stride[i];
    rows = 1;
  }
  return Region{s.base, (uintptr_t)rows, (uintptr_t)width, (uintptr_t)(rows == 1 ? width : pitch)};
}

// Do two runs of a nested shape, `delta` bytes apart, meet for some steps along axes 0 .. axis of either?
bool runs_meet(const PoolShape& s, int axis, int64_t delta) {
  if (axis < 0) return delta < s.width && -delta < s.width;
  // all that lies inside a stride is no longer than it, so only the two steps that leave less than a stride can do
  const int64_t q = delta >= 0 ? delta / s.stride[axis] : -((-delta + s.stride[axis] - 1) / s.stride[axis]);
  for (int64_t step = q; step <= q + 1; ++step)
    if (step < s.n[axis] && -step < s.n[axis] && runs_meet(s, axis - 1, delta - step * s.stride[axis])) return true;
  return false;
}

// Exact where both sides lie alike, as halves of one buffer do; otherwise by their regions.
bool pools_meet(const PoolShape& a, const PoolShape& b) {
  bool alike = a.nested && b.nested && a.axes == b.axes;
  for (int i = 0; alike && i < a.axes; ++i) alike = a.stride[i] == b.stride[i] && a.n[i] == b.n[i];
  return alike ? runs_meet(a, a.axes - 1, (int64_t)(b.base - a.base)) : may_overlap(pool_region(a), pool_region(b));
}

// One side of a paged cache: strides and alignment.
int check_cache_side(const qknorm_paged_cache& c, void* base, int64_t page, int64_t token, int64_t head, Region* region, bool* vec16,
                     bool* vec8) {
  const uintptr_t eb = c.e4m3 ? 1 : 2;
  if (c.num_pages > 0 && !base) return QKNORM_ERR_NULL;
  if (page < 0 || token < 0 || head < 0) return QKNORM_ERR_SHAPE;
  if (c.num_pages == 0) {  // an empty pool: nothing in it is ever touched
    *region = Region{0, 0, 0, 0};
    *vec16 = *vec8 = true;
    return QKNORM_OK;
  }
  // no two elements of a page in the same place: heads inside a token's stride or tokens inside a head's
  const int64_t d = c.head_dim;
  if (c.heads > 1 && head < d) return QKNORM_ERR_SHAPE;
  if (c.page_size > 1 && token < d) return QKNORM_ERR_SHAPE;
  if (c.heads > 1 && c.page_size > 1 && (__int128)token < (__int128)(c.heads - 1) * head + d &&
      (__int128)head < (__int128)(c.page_size - 1) * token + d)
    return QKNORM_ERR_SHAPE;
  const __int128 total = (__int128)(c.num_pages > 1 ? c.num_pages - 1 : 0) * page + (__int128)(c.page_size - 1) * token +
                         (__int128)(c.heads - 1) * head + d;
  if (total > ((__int128)1 << 60)) return QKNORM_ERR_SHAPE;
  if (c.num_pages > 1 && page < d) return QKNORM_ERR_SHAPE;
  if (((uintptr_t)base) % eb != 0) return QKNORM_ERR_ALIGN;
  *region = pool_region(pool_shape(c, base, page, token, head));
  const uintptr_t all = (uintptr_t)base | ((uintptr_t)page * eb) | ((uintptr_t)token * eb) | ((uintptr_t)head * eb);
  *vec16 = all % 16 == 0;
  *vec8 = all % 8 == 0;
  return QKNORM_OK;
}

struct CacheFacts {
  Region k, v;
  bool vec16, vec8;
};

int check_cache(const qknorm_paged_cache* c, CacheFacts* f) {
  if (!c) return QKNORM_ERR_NULL;
  if (c->num_pages < 0 || c->num_pages > 0x7fffffff || c->page_size < 1 || c->heads < 1) return QKNORM_ERR_SHAPE;
  if (c->head_dim < 1 || c->head_dim > QKNORM_MAX_HEAD_DIM) return QKNORM_ERR_HEADS;
  if ((int64_t)c->heads * c->head_dim > kMaxDim) return QKNORM_ERR_SHAPE;
  if (c->e4m3 != 0 && c->e4m3 != 1) return QKNORM_ERR_SHAPE;
  if (c->e4m3 && (!(c->k_scale > 0.0f) || !isfinite(c->k_scale) || !(c->v_scale > 0.0f) || !isfinite(c->v_scale))) return QKNORM_ERR_SHAPE;
  bool k16, k8, v16, v8;
  int rc = check_cache_side(*c, c->k, c->k_page, c->k_token, c->k_head, &f->k, &k16, &k8);
  if (rc != QKNORM_OK) return rc;
  rc = check_cache_side(*c, c->v, c->v_page, c->v_token, c->v_head, &f->v, &v16, &v8);
  if (rc != QKNORM_OK) return rc;
  f->vec16 = k16 && v16;
  f->vec8 = k8 && v8;
  return QKNORM_OK;
}

// A 4-bit cache: codes of K, of V, scales of K, of V.
struct E2m1Facts {
  Region region[4];
  PoolShape shape[4];
  bool vec16;  // 16-byte copies of the codes
};

// One side of it, in bytes, as check_cache_side and pool_shape look at it.
qknorm_paged_cache e2m1_side(const qknorm_paged_cache_e2m1& c, int i) {
  qknorm_paged_cache s = {};
  s.num_pages = c.num_pages;
  s.page_size = c.page_size;
  s.heads = c.heads;
  s.head_dim = i < 2 ? c.head_dim / 2 : c.head_dim / 16;
  s.e4m3 = 1;
  s.k = i == 0 ? c.k : i == 1 ? c.v : i == 2 ? c.k_scales : c.v_scales;
  s.k_page = i == 0 ? c.k_page : i == 1 ? c.v_page : i == 2 ? c.ks_page : c.vs_page;
  s.k_token = i == 0 ? c.k_token : i == 1 ? c.v_token : i == 2 ? c.ks_token : c.vs_token;
  s.k_head = i == 0 ? c.k_head : i == 1 ? c.v_head : i == 2 ? c.ks_head : c.vs_head;
  return s;
}

int check_cache(const qknorm_paged_cache_e2m1* c, E2m1Facts* f) {
  if (!c) return QKNORM_ERR_NULL;
  if (c->num_pages < 0 || c->num_pages > 0x7fffffff || c->page_size < 1 || c->heads < 1) return QKNORM_ERR_SHAPE;
  if (c->head_dim < 16 || c->head_dim > QKNORM_MAX_HEAD_DIM_E2M1 || c->head_dim % 16 != 0) return QKNORM_ERR_HEADS;
  if ((int64_t)c->heads * c->head_dim > kMaxDim) return QKNORM_ERR_SHAPE;
  if (!(c->k_scale > 0.0f) || !isfinite(c->k_scale) || !(c->v_scale > 0.0f) || !isfinite(c->v_scale)) return QKNORM_ERR_SHAPE;
  f->vec16 = c->head_dim % 32 == 0;
  const int blocks = c->head_dim / 16;
  const uintptr_t low = blocks & -blocks, unit = low > 8 ? 8 : low;
  for (int i = 0; i < 4; ++i) {
    const qknorm_paged_cache s = e2m1_side(*c, i);
    bool v16, v8;
    const int rc = check_cache_side(s, s.k, s.k_page, s.k_token, s.k_head, &f->region[i], &v16, &v8);
    if (rc != QKNORM_OK) return rc;
    f->shape[i] = pool_shape(s, s.k, s.k_page, s.k_token, s.k_head);
    if (c->num_pages == 0) continue;
    const uintptr_t all = (uintptr_t)s.k | (uintptr_t)s.k_page | (uintptr_t)s.k_token | (uintptr_t)s.k_head;
    if (i < 2 ? !v8 : all % unit != 0) return QKNORM_ERR_ALIGN;
    if (i < 2) f->vec16 = f->vec16 && v16;
  }
  return QKNORM_OK;
}

// Launches R (everything but the launch shape filled in).  cache_bytes 0: no cache.  vec: the vector kernel's alignment holds.
int launch_rope(RopeParams& R, int elem_bytes, int cache_bytes, int norm, bool vec, cudaStream_t stream) {
  const DeviceInfo* dev = nullptr;
  int rc = current_device(&dev);
  if (rc != QKNORM_OK) return rc;
  const char* force = env_str("QKNORM_FORCE_VARIANT");
  if (force && strcmp(force, "general") == 0) vec = false;
  if (vec) {
    R.log_lph = 0;
    while ((16 << R.log_lph) < R.head_dim) ++R.log_lph;
    const int heads = R.q.heads + R.k.heads + (cache_bytes ? R.v.heads : 0);
    R.slots_per_token = heads << R.log_lph;
    // Few tokens: one unit per thread, for latency.  Many: four, which spread a thread's start (which head, which rows) and the
    // token's barrier over more elements -- 16384 tokens of 5120 + 1024 + 1024 take 154 us with one, 103 with two, 92 with four.
    int upt = R.T < 2 * dev->sm_count ? 1 : 4;
    if (R.slots_per_token > 1024) upt = 4;
    if (R.slots_per_token <= 4096) {
      R.threads_per_token = round_up((R.slots_per_token + upt - 1) / upt, 32);
      // short rows: several tokens share a CTA of about 128 threads
      R.tokens_per_cta = R.T >= 2 * dev->sm_count && R.threads_per_token < 128 ? 128 / R.threads_per_token : 1;
      const int smem = R.tokens_per_cta * R.rot_dim * (int)sizeof(float2) / 2;
      RopeKernel fn = rope_kernel_for(elem_bytes, cache_bytes, norm, R.interleaved != 0, upt, R.tokens_per_cta * R.threads_per_token);
      const long long grid = (R.T + R.tokens_per_cta - 1) / R.tokens_per_cta;
      if (grid <= 0x7fffffff) {
        const cudaError_t e = launch_overlapped(fn, (unsigned)grid, (unsigned)(R.tokens_per_cta * R.threads_per_token), (size_t)smem, stream, R);
        if (e != cudaSuccess) return set_cuda_error(e);
        return finish_launch(cache_bytes ? "append" : "rope");
      }
    }
  }
  RopeGeneralKernel gen = rope_general_kernel_for(elem_bytes, cache_bytes);
  int bres = 1;
  rc = resident_blocks((const void*)gen, kRopeGeneralThreads, 0, &bres);
  if (rc != QKNORM_OK) return rc;
  long long grid = (long long)bres * dev->sm_count;
  if (grid > R.T) grid = R.T;
  const cudaError_t e = launch_overlapped(gen, (unsigned)grid, (unsigned)kRopeGeneralThreads, 0, stream, R, norm);
  if (e != cudaSuccess) return set_cuda_error(e);
  return finish_launch(cache_bytes ? "append_general" : "rope_general");
}

template <class Rotation>
int run_rope(int elem_bytes, const void* q, const void* k, const Rotation* rot, int64_t T, int32_t dq, int32_t dk,
             int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* oq, void* ok, int64_t ld_oq, int64_t ld_ok,
             cudaStream_t stream) {
  if (T < 0 || dq < 0 || dk < 0 || dq > kMaxDim || dk > kMaxDim) return QKNORM_ERR_SHAPE;
  if (head_dim < 1 || head_dim > QKNORM_MAX_HEAD_DIM || dq % head_dim != 0 || dk % head_dim != 0) return QKNORM_ERR_HEADS;
  if (inverse != 0 && inverse != 1) return QKNORM_ERR_SHAPE;
  if (!rot) return QKNORM_ERR_NULL;
  RopeParams R;
  memset(&R, 0, sizeof(R));
  int rc;
  if ((rc = row_stride(ld_q, dq, &R.q.ldx)) || (rc = row_stride(ld_k, dk, &R.k.ldx)) || (rc = row_stride(ld_oq, dq, &R.q.ldy)) ||
      (rc = row_stride(ld_ok, dk, &R.k.ldy)))
    return rc;
  if (T == 0) return QKNORM_OK;
  if (dq == 0 && dk == 0) return QKNORM_ERR_SHAPE;
  if ((rc = check_rotation(rot, head_dim, R, T)) != QKNORM_OK) return rc;
  if (inverse) R.turns_sign = -R.turns_sign;
  R.T = T;
  R.head_dim = head_dim;
  CallRegions c;
  uintptr_t vec = (uintptr_t)head_dim | (uintptr_t)R.rot_dim;  // multiples of 16, checked together
  const uintptr_t eb = (uintptr_t)elem_bytes, unit = 8 * eb;
  bool aligned = vec % 16 == 0;
  struct Side {
    RopeSide* s;
    const void* x;
    void* y;
    int d;
  } sides[2] = {{&R.q, q, oq, dq}, {&R.k, k, ok, dk}};
  for (Side& sd : sides) {
    if (sd.d == 0) continue;
    if (!sd.x || !sd.y) return QKNORM_ERR_NULL;
    if ((((uintptr_t)sd.x) | ((uintptr_t)sd.y)) % eb != 0) return QKNORM_ERR_ALIGN;
    sd.s->x = sd.x;
    sd.s->y = sd.y;
    sd.s->heads = sd.d / head_dim;
    aligned = aligned && (((uintptr_t)sd.x) | ((uintptr_t)sd.y) | ((uintptr_t)sd.s->ldx * eb) | ((uintptr_t)sd.s->ldy * eb)) % unit == 0;
    c.own[c.outs] = c.ins;
    c.out[c.outs++] = Region{(uintptr_t)sd.y, (uintptr_t)T, (uintptr_t)sd.d * eb, (uintptr_t)sd.s->ldy * eb};
    c.in[c.ins++] = Region{(uintptr_t)sd.x, (uintptr_t)T, (uintptr_t)sd.d * eb, (uintptr_t)sd.s->ldx * eb};
  }
  rotation_regions(R, c);
  if ((rc = check_regions(c)) != QKNORM_OK) return rc;
  return launch_rope(R, elem_bytes, 0, kNormNone, aligned, stream);
}

// What an append needs to know of a cache: its sides, 2 of them or (with a 4-bit cache's scales) 4.
struct AppendCache {
  int bytes, sides;  // bytes: of an element, or kCacheE2m1
  CacheSide side[4];
  Region region[4];
  PoolShape shape[4];
  bool vec;
};

int append_cache(const qknorm_paged_cache* c, AppendCache* a) {
  CacheFacts f;
  const int rc = check_cache(c, &f);
  if (rc != QKNORM_OK) return rc;
  a->bytes = c->e4m3 ? 1 : 2;
  a->sides = 2;
  a->side[0] = CacheSide{c->k, c->k_page, c->k_token, c->k_head, c->e4m3 ? 1.0f / c->k_scale : 1.0f};
  a->side[1] = CacheSide{c->v, c->v_page, c->v_token, c->v_head, c->e4m3 ? 1.0f / c->v_scale : 1.0f};
  a->region[0] = f.k;
  a->region[1] = f.v;
  if (c->num_pages > 0) {
    a->shape[0] = pool_shape(*c, c->k, c->k_page, c->k_token, c->k_head);
    a->shape[1] = pool_shape(*c, c->v, c->v_page, c->v_token, c->v_head);
  }
  a->vec = c->e4m3 ? f.vec8 : f.vec16;
  return QKNORM_OK;
}

int append_cache(const qknorm_paged_cache_e2m1* c, AppendCache* a) {
  E2m1Facts f;
  const int rc = check_cache(c, &f);
  if (rc != QKNORM_OK) return rc;
  a->bytes = kCacheE2m1;
  a->sides = 4;
  for (int i = 0; i < 4; ++i) {
    const qknorm_paged_cache s = e2m1_side(*c, i);
    a->side[i] = CacheSide{s.k, s.k_page, s.k_token, s.k_head, i == 0 ? 1.0f / c->k_scale : i == 1 ? 1.0f / c->v_scale : 1.0f};
    a->region[i] = f.region[i];
    a->shape[i] = f.shape[i];
  }
  a->vec = true;  // what a vector store needs, check_cache has asked for
  return QKNORM_OK;
}

template <class Rotation, class Cache>
int run_append(const void* q, const void* k, const void* v, const void* gq, const void* gk, int32_t norm, float eps,
               const Rotation* rot, const int64_t* slots, const Cache* cache, int64_t T, int32_t dq, int64_t ld_q,
               int64_t ld_k, int64_t ld_v, void* oq, int64_t ld_oq, cudaStream_t stream) {
  AppendCache f;
  int rc = append_cache(cache, &f);
  if (rc != QKNORM_OK) return rc;
  const int hd = cache->head_dim, dk = cache->heads * hd;
  if (T < 0 || dq < 0 || dq > kMaxDim) return QKNORM_ERR_SHAPE;
  if (dq % hd != 0) return QKNORM_ERR_HEADS;
  if (norm < kNormNone || norm > kNormHead) return QKNORM_ERR_SHAPE;
  if (norm != kNormNone && !(eps >= 0.0f)) return QKNORM_ERR_EPS;
  if (!isfinite(f.side[0].inv_scale) || !isfinite(f.side[1].inv_scale)) return QKNORM_ERR_SHAPE;
  RopeParams R;
  memset(&R, 0, sizeof(R));
  if ((rc = row_stride(ld_q, dq, &R.q.ldx)) || (rc = row_stride(ld_oq, dq, &R.q.ldy)) || (rc = row_stride(ld_k, dk, &R.k.ldx)) ||
      (rc = row_stride(ld_v, dk, &R.v.ldx)))
    return rc;
  if (T == 0) return QKNORM_OK;
  if ((rc = check_rotation(rot, hd, R, T)) != QKNORM_OK) return rc;
  if (!k || !v || !slots || (norm != kNormNone && !gk)) return QKNORM_ERR_NULL;
  if (dq > 0 && (!q || !oq || (norm != kNormNone && !gq))) return QKNORM_ERR_NULL;
  uintptr_t ptrs = (uintptr_t)k | (uintptr_t)v, strides = (uintptr_t)R.k.ldx | (uintptr_t)R.v.ldx;
  if (norm != kNormNone) ptrs |= (uintptr_t)gk;
  if (dq > 0) {
    ptrs |= (uintptr_t)q | (uintptr_t)oq;
    strides |= (uintptr_t)R.q.ldx | (uintptr_t)R.q.ldy;
    if (norm != kNormNone) ptrs |= (uintptr_t)gq;
  }
  if (ptrs & 1u) return QKNORM_ERR_ALIGN;
  if (((uintptr_t)slots) & 7u) return QKNORM_ERR_ALIGN;
  R.T = T;
  R.head_dim = hd;
  R.inv_hd = 1.0f / (float)hd;
  R.eps = eps;
  if (dq > 0) {
    R.q.x = q;
    R.q.y = oq;
    R.q.gamma = (const uint16_t*)gq;
    R.q.heads = dq / hd;
    R.q.inv_d = 1.0f / (float)dq;
  }
  R.k.x = k;
  R.k.gamma = (const uint16_t*)gk;
  R.k.heads = R.v.heads = cache->heads;
  R.k.inv_d = 1.0f / (float)dk;
  R.v.x = v;
  R.ck = f.side[0];
  R.cv = f.side[1];
  if (f.sides == 4) {
    R.cks = f.side[2];
    R.cvs = f.side[3];
  }
  R.slots = (const long long*)slots;
  R.num_slots = (long long)cache->num_pages * cache->page_size;
  R.page_size = cache->page_size;
  R.page_shift = log2_or_minus_one(cache->page_size);
  const uintptr_t rows = (uintptr_t)T, qb = (uintptr_t)dq * 2, kb = (uintptr_t)dk * 2;
  CallRegions c;
  if (dq > 0) {
    c.own[0] = 0;
    c.out[c.outs++] = Region{(uintptr_t)oq, rows, qb, (uintptr_t)R.q.ldy * 2};
    c.in[c.ins++] = Region{(uintptr_t)q, rows, qb, (uintptr_t)R.q.ldx * 2};
    if (norm != kNormNone) c.in[c.ins++] = flat(gq, qb);
  }
  c.pools = c.outs;
  c.num_pools = f.sides;
  for (int i = 0; i < f.sides; ++i) {
    c.own[c.outs] = -1;
    c.out[c.outs++] = f.region[i];
  }
  c.in[c.ins++] = Region{(uintptr_t)k, rows, kb, (uintptr_t)R.k.ldx * 2};
  c.in[c.ins++] = Region{(uintptr_t)v, rows, kb, (uintptr_t)R.v.ldx * 2};
  if (norm != kNormNone) c.in[c.ins++] = flat(gk, kb);
  c.in[c.ins++] = flat(slots, 8 * rows);
  rotation_regions(R, c);
  if ((rc = check_regions(c)) != QKNORM_OK) return rc;
  if (cache->num_pages > 0)
    for (int i = 0; i < f.sides; ++i)
      for (int j = 0; j < i; ++j)
        if (pools_meet(f.shape[i], f.shape[j])) return QKNORM_ERR_ALIAS;
  bool vec = (hd | R.rot_dim) % 16 == 0 && ptrs % 16 == 0 && strides % 8 == 0 && f.vec;
  // a block of 16 elements lies with two neighbouring lanes in the half layout: both have to be of the part that turns
  if (f.bytes == kCacheE2m1 && R.rot_dim % 32 != 0 && !R.interleaved) vec = false;
  return launch_rope(R, 2, f.bytes, norm, vec, stream);
}

// ---- attention over the paged cache ---------------------------------------------------------------

AttnTcKernel attn_tc_for(int dp, AttnFormat format, int form, bool tma, int* smem) {
  if (format == kAttnE4m3) return dp == 64 ? attn_tc_kernel_e4m364(form, tma, smem) : attn_tc_kernel_e4m3128(form, tma, smem);
  if (format == kAttnWidened) return dp == 64 ? attn_tc_kernel_wide64(form, tma, smem) : attn_tc_kernel_wide128(form, tma, smem);
  return dp == 64 ? attn_tc_kernel_bf1664(form, tma, smem) : attn_tc_kernel_bf16128(form, tma, smem);
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, looked up once; nullptr if it cannot be had.
EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return (EncodeTiled)p;
  }();
  return fn;
}

// How copies can take a whole head of 128 bf16 values: both sides have to allow it.
int whole_head_kind(const qknorm_paged_cache& c) {
  if (c.e4m3 || c.head_dim != 128) return kBoxHalf;
  if ((c.heads == 1 || (c.k_head == 128 && c.v_head == 128))) return kBoxHeadInRow;
  if ((c.num_pages == 1 || (c.k_page == c.heads * c.k_head && c.v_page == c.heads * c.v_head)) && c.num_pages * c.heads < 0x7fffffff)
    return kBoxHeadInPage;
  return kBoxHalf;
}

// One side of the cache, laid out as `kind` says; a copy takes `rows` tokens, swizzled as the matrix unit reads them (FP8: as
// they are, to be widened).  False: no such map.
bool encode_side(CUtensorMap* map, const qknorm_paged_cache& c, const AttnSide& s, int kind, int dp, int rows) {
  const EncodeTiled enc = encode_tiled();
  if (!enc) return false;
  const cuuint64_t eb = c.e4m3 ? 1 : 2;
  // the stride of an axis of one is never used, but has to look like one
  const cuuint64_t row = ((cuuint64_t)c.head_dim * eb + 15) / 16 * 16;
  const cuuint64_t token = c.page_size > 1 ? s.token * eb : row, head = c.heads > 1 ? s.head * eb : row, page = c.num_pages > 1 ? s.page * eb : row;
  const cuuint64_t pages = (cuuint64_t)c.num_pages, heads = (cuuint64_t)c.heads, tokens = (cuuint64_t)c.page_size;
  cuuint64_t dims[5], strides[4];
  cuuint32_t box[5];
  cuuint32_t n = 4;
  if (kind == kBoxHalf) {
    const cuuint64_t d[4] = {(cuuint64_t)c.head_dim, tokens, heads, pages}, st[3] = {token, head, page};
    const cuuint32_t b[4] = {(cuuint32_t)(c.e4m3 ? dp : 64), (cuuint32_t)rows, 1, 1};
    memcpy(dims, d, sizeof(d));
    memcpy(strides, st, sizeof(st));
    memcpy(box, b, sizeof(b));
  } else {
    n = 5;
    const bool in_row = kind == kBoxHeadInRow;
    const cuuint64_t d[5] = {64, 8, in_row ? 2 * heads : 2, tokens / 8, in_row ? pages : pages * heads};
    const cuuint64_t st[4] = {token, 128, 8 * token, in_row ? page : c.heads > 1 ? head : page};
    const cuuint32_t b[5] = {64, 8, 2, (cuuint32_t)rows / 8, 1};
    memcpy(dims, d, sizeof(d));
    memcpy(strides, st, sizeof(st));
    memcpy(box, b, sizeof(b));
  }
  for (cuuint32_t i = 0; i + 1 < n; ++i)
    if (strides[i] == 0 || strides[i] % 16 != 0 || strides[i] >= ((cuuint64_t)1 << 40)) return false;
  const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
  return enc(map, c.e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, n, const_cast<void*>(s.base), dims, strides, box,
             ones, CU_TENSOR_MAP_INTERLEAVE_NONE, c.e4m3 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The tensor-core kernel hands registers from its loaders to its softmax warps: it must have been compiled to start with the
// number the split adds up to, or the warps that ask for more would wait for ever.
int attn_tc_registers_ok(const void* fn) {
  static const void* known[32];
  static int n = 0;
  std::lock_guard<std::mutex> lock(g_occ_mutex);
  for (int i = 0; i < n; ++i)
    if (known[i] == fn) return QKNORM_OK;
  cudaFuncAttributes a;
  const cudaError_t e = cudaFuncGetAttributes(&a, fn);
  if (e != cudaSuccess) return set_cuda_error(e);
  if (a.numRegs != kAttnTcRegs) return set_cuda_error(cudaErrorLaunchOutOfResources);
  if (n < 32) known[n++] = fn;
  return QKNORM_OK;
}

// q as [token][head][d]; a copy takes `tokens` tokens of the `group` query heads of a key head and 64 columns.
bool encode_q(CUtensorMap* map, const AttnParams& P, int tokens) {
  const EncodeTiled enc = encode_tiled();
  if (!enc) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)P.head_dim, (cuuint64_t)P.heads_q, (cuuint64_t)P.T};
  const cuuint64_t strides[2] = {(cuuint64_t)P.head_dim * 2, (cuuint64_t)P.ld_q * 2};
  if (strides[0] % 16 != 0 || strides[1] % 16 != 0 || strides[1] >= ((cuuint64_t)1 << 40)) return false;
  const cuuint32_t box[3] = {64, (cuuint32_t)P.group, (cuuint32_t)tokens};
  const cuuint32_t ones[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t*>(P.q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a call is cut: sizes only, so that the workspace can be asked for beforehand.
struct AttnPlan {
  bool tc = false;
  int form = kAttnTwo;
  int tok_per_tile = 1, tiles_per_item = 1, q_items = 1, grid = 1, part_rows = 0;
  int own = 1;
  bool cuts = false;  // some unit may be cut between CTAs
};

AttnPlan plan_attn(int seqs, int64_t T, int max_q, int64_t max_keys, int heads_q, int heads_kv, int head_dim, bool causal, int window,
                   int sms) {
  AttnPlan p;
  const int group = heads_q / heads_kv;
  p.tc = head_dim % 8 == 0 && head_dim <= 128 && group <= kAttnTile;
  if (!p.tc) return p;
  p.tok_per_tile = kAttnTile / group;
  if ((int64_t)max_q > T) max_q = (int)T;
  p.tiles_per_item = max_q <= p.tok_per_tile ? 1 : 2;
  p.form = p.tiles_per_item == 2 ? kAttnTwo : max_q * group <= 32 ? kAttnQuad : kAttnOne;
  const int per_item = p.tok_per_tile * p.tiles_per_item;
  p.q_items = (max_q + per_item - 1) / per_item;
  int64_t tiles = (max_keys + kAttnTile - 1) / kAttnTile;  // of a unit, at most
  if (window > 0) {
    // its first row's window, and the keys that its later rows see beyond: as many as there are rows -- or, without the causal edge, all
    // up to the sequence's end, which the sequence's first unit has the most of
    const int64_t span = ((int64_t)window + (causal ? per_item : max_q) - 1 + kAttnTile - 2) / kAttnTile + 1;
    if (span < tiles) tiles = span;
  }
  // One CTA per SM, and none for less than two tiles.  Units that a batch of T rows can have:
  int64_t pieces = (int64_t)p.q_items * seqs;
  if (T / per_item + seqs < pieces) pieces = T / per_item + seqs;
  // What a unit's start and end take, in tiles.  Two query tiles, a prompt of 8192: 1106 us with 1, 928 with 2, 897 with 3, 853 with 4,
  // 852 with 5; one query tile: no difference between 1 and 5.
  p.own = p.tiles_per_item == 1 ? 1 : 4;
  const double all = (double)pieces * heads_kv * (double)(tiles + p.own);
  p.grid = all >= 2.0 * sms ? sms : (int)((all + 1.0) / 2.0);
  // no cut can fall inside a unit of at most twice the distance at which cuts move to its ends; shares are at most this long
  const int longest = tiles + p.own < 0x3fffffff ? (int)(tiles + p.own) : 0x3fffffff;
  p.cuts = longest > 2 * attn_snap((int64_t)(all / p.grid) + 1, p.own, longest);
  p.part_rows = p.form == kAttnQuad ? 32 : kAttnTile * p.tiles_per_item;
  return p;
}

// Can the kernel count the call's items in 32 bits?
bool attn_countable(const AttnPlan& p, int seqs, int heads_kv) { return (int64_t)p.q_items * seqs <= 0x3fffffff && (int64_t)seqs * heads_kv <= 0x3fffffff; }

// starts, then parts' rows, then their log-sums
int64_t attn_starts_bytes(const AttnPlan& p) { return p.cuts ? (int64_t)p.grid * 32 : 0; }
int64_t attn_parts(const AttnPlan& p) { return p.cuts ? (int64_t)p.grid * 2 * p.part_rows : 0; }
int64_t attn_workspace(const AttnPlan& p, int head_dim) {
  if (!p.tc) return 0;
  return (attn_starts_bytes(p) + attn_parts(p) * (head_dim + 1) * 4 + 15) / 16 * 16;
}

int check_attn_sizes(int32_t seqs, int64_t T, int32_t max_q, int32_t max_kv, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                     int32_t window) {
  if (seqs < 0 || seqs > 0x3fffffff || T < 0 || T > 0x7fffffff || max_q < 0 || max_kv < 0 || max_kv > QKNORM_MAX_KEYS || window < 0) return QKNORM_ERR_SHAPE;
  if (head_dim < 1 || head_dim > QKNORM_MAX_HEAD_DIM) return QKNORM_ERR_HEADS;
  if (heads_q < 1 || heads_kv < 1 || heads_q % heads_kv != 0) return QKNORM_ERR_HEADS;
  if ((int64_t)heads_q * head_dim > kMaxDim) return QKNORM_ERR_SHAPE;
  return QKNORM_OK;
}

int run_attn_workspace(int32_t seqs, int64_t T, int32_t max_q, int32_t max_kv, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                       int32_t window, int64_t* bytes) {
  if (!bytes) return QKNORM_ERR_NULL;
  int rc = check_attn_sizes(seqs, T, max_q, max_kv, heads_q, heads_kv, head_dim, window);
  if (rc != QKNORM_OK) return rc;
  *bytes = 0;
  if (seqs == 0 || T == 0 || max_q == 0) return QKNORM_OK;
  const DeviceInfo* dev = nullptr;
  rc = current_device(&dev);
  if (rc != QKNORM_OK) return rc;
  for (const bool causal : {true, false}) {  // enough for either
    const int64_t need = attn_workspace(plan_attn(seqs, T, max_q, max_kv, heads_q, heads_kv, head_dim, causal, window, dev->sm_count), head_dim);
    if (need > *bytes) *bytes = need;
  }
  return QKNORM_OK;
}

// widened: a 4-bit cache's codes times their scales, V in fp16, though `cache` says bf16; V is multiplied by v_scale (an FP8 cache has its own).
int run_attn(const void* q, int64_t ld_q, const qknorm_paged_cache* cache, const int32_t* table, int32_t table_cols, int64_t ld_table,
             const int32_t* kv_lens, const int32_t* q_starts, int32_t seqs, int64_t T, int32_t max_q, int32_t max_kv, int32_t heads_q,
             float scale, int32_t causal, int32_t window, void* out, int64_t ld_out, float* lse, void* ws, int64_t ws_bytes,
             cudaStream_t stream, bool widened = false, float v_scale = 1.0f) {
  CacheFacts f;
  int rc = check_cache(cache, &f);
  if (rc != QKNORM_OK) return rc;
  rc = check_attn_sizes(seqs, T, max_q, max_kv, heads_q, cache->heads, cache->head_dim, window);
  if (rc != QKNORM_OK) return rc;
  if (!(scale > 0.0f) || !isfinite(scale)) return QKNORM_ERR_SHAPE;
  const float c = (float)((double)scale * (cache->e4m3 ? cache->k_scale : 1.0f) * 1.44269504088896340736);
  if (!isfinite(c)) return QKNORM_ERR_SHAPE;
  if (causal != 0 && causal != 1) return QKNORM_ERR_SHAPE;
  if (table_cols < 0 || ld_table < 0 || (ld_table != 0 && ld_table < table_cols)) return QKNORM_ERR_SHAPE;
  AttnParams P;
  memset(&P, 0, sizeof(P));
  const int d = heads_q * cache->head_dim;
  if ((rc = row_stride(ld_q, d, &P.ld_q)) || (rc = row_stride(ld_out, d, &P.ld_out))) return rc;
  if (seqs == 0 || T == 0 || max_q == 0) return QKNORM_OK;
  if (!q || !out || !kv_lens || !q_starts || (table_cols > 0 && !table)) return QKNORM_ERR_NULL;
  if ((((uintptr_t)q) | ((uintptr_t)out)) & 1u) return QKNORM_ERR_ALIGN;
  if ((((uintptr_t)table) | ((uintptr_t)kv_lens) | ((uintptr_t)q_starts) | ((uintptr_t)lse)) & 3u) return QKNORM_ERR_ALIGN;

  const DeviceInfo* dev = nullptr;
  rc = current_device(&dev);
  if (rc != QKNORM_OK) return rc;
  const AttnFormat format = widened ? kAttnWidened : cache->e4m3 ? kAttnE4m3 : kAttnBf16;
  AttnPlan plan = plan_attn(seqs, T, max_q, max_kv, heads_q, cache->heads, cache->head_dim, causal != 0, window, dev->sm_count);
  const bool aligned = (((uintptr_t)q) | ((uintptr_t)out) | ((uintptr_t)P.ld_q * 2) | ((uintptr_t)P.ld_out * 2)) % 16 == 0 && f.vec16 &&
                       (!cache->e4m3 || cache->head_dim % 16 == 0);
  const char* force = env_str("QKNORM_FORCE_VARIANT");
  if (!aligned || (force && strcmp(force, "general") == 0)) plan.tc = false;
  const int64_t need = attn_workspace(plan, cache->head_dim);
  if (need > 0) {
    if (!ws || ws_bytes < need || !aligned16(ws)) return QKNORM_ERR_SCRATCH;
    const Region w = flat(ws, (uintptr_t)need);
    const Region others[] = {Region{(uintptr_t)q, (uintptr_t)T, (uintptr_t)d * 2, (uintptr_t)P.ld_q * 2},
                             Region{(uintptr_t)out, (uintptr_t)T, (uintptr_t)d * 2, (uintptr_t)P.ld_out * 2},
                             f.k, f.v,
                             Region{(uintptr_t)table, (uintptr_t)seqs, (uintptr_t)table_cols * 4, (uintptr_t)(ld_table ? ld_table : table_cols) * 4},
                             flat(kv_lens, 4 * (uintptr_t)seqs), flat(q_starts, 4 * ((uintptr_t)seqs + 1)),
                             flat(lse, lse ? 4 * (uintptr_t)T * heads_q : 0)};
    for (const Region& o : others)
      if (may_overlap(w, o)) return QKNORM_ERR_SCRATCH;
  }
  {
    // q and out stay apart: copies of q's rows bring along rows of other sequences, whose results may be written already
    CallRegions c;
    c.own[c.outs] = -1;
    c.out[c.outs++] = Region{(uintptr_t)out, (uintptr_t)T, (uintptr_t)d * 2, (uintptr_t)P.ld_out * 2};
    if (lse) {
      c.own[c.outs] = -1;
      c.out[c.outs++] = flat(lse, 4 * (uintptr_t)T * heads_q);
    }
    c.in[c.ins++] = Region{(uintptr_t)q, (uintptr_t)T, (uintptr_t)d * 2, (uintptr_t)P.ld_q * 2};
    c.in[c.ins++] = f.k;
    c.in[c.ins++] = f.v;
    if (table_cols > 0)
      c.in[c.ins++] = Region{(uintptr_t)table, (uintptr_t)seqs, (uintptr_t)table_cols * 4, (uintptr_t)(ld_table ? ld_table : table_cols) * 4};
    c.in[c.ins++] = flat(kv_lens, 4 * (uintptr_t)seqs);
    c.in[c.ins++] = flat(q_starts, 4 * ((uintptr_t)seqs + 1));
    if ((rc = check_regions(c)) != QKNORM_OK) return rc;
  }

  P.q = (const uint16_t*)q;
  P.out = (uint16_t*)out;
  P.k = AttnSide{cache->k, cache->k_page, cache->k_token, cache->k_head};
  P.v = AttnSide{cache->v, cache->v_page, cache->v_token, cache->v_head};
  if (cache->num_pages == 0) P.k = P.v = AttnSide{(const void*)((uintptr_t)q & ~(uintptr_t)15), 0, 0, 0};  // never read, but copies of no bytes name it
  P.num_pages = cache->num_pages;
  P.page_size = cache->page_size;
  P.page_shift = log2_or_minus_one(cache->page_size);
  P.table = table;
  P.ld_table = ld_table ? ld_table : table_cols;
  P.kv_lens = kv_lens;
  P.q_starts = q_starts;
  P.seqs = seqs;
  P.T = T;
  P.max_q = (int64_t)max_q < T ? max_q : (int)T;
  P.max_keys = (int64_t)table_cols * cache->page_size < max_kv ? (int64_t)table_cols * cache->page_size : max_kv;
  P.heads_q = heads_q;
  P.heads_kv = cache->heads;
  P.group = heads_q / cache->heads;
  P.head_dim = cache->head_dim;
  P.c = fmaxf(c, kAttnLeastC);
  P.v_scale = cache->e4m3 ? cache->v_scale : v_scale;
  P.causal = causal;
  P.window = window;
  P.lse = lse;
  P.tok_per_tile = plan.tok_per_tile;
  P.tiles_per_item = plan.tiles_per_item;
  P.q_items = plan.q_items;
  P.grid = plan.grid;
  P.part_rows = plan.part_rows;
  P.own = plan.own;
  const int wait_us = env_int("QKNORM_ATTN_WAIT_US", 2000000);  // shorter in tests of the waits
  P.wait_ns = 1000u * (unsigned)(wait_us < 1 ? 1 : wait_us > 2000000 ? 2000000 : wait_us);
  P.error = dev->ring_error;
  if (plan.tc && plan.cuts) {
    P.starts = (int*)ws;
    P.part_o = (float*)((char*)ws + attn_starts_bytes(plan));
    P.part_z = P.part_o + attn_parts(plan) * cache->head_dim;
  }

  if (!plan.tc) {
    AttnKernel gen = attn_general_kernel_for(format);
    int bres = 1;
    rc = resident_blocks((const void*)gen, kAttnGeneralThreads, 0, &bres);
    if (rc != QKNORM_OK) return rc;
    long long grid = (long long)bres * dev->sm_count;
    const long long want = ((long long)seqs * P.max_q * heads_q + kAttnGeneralThreads / 32 - 1) / (kAttnGeneralThreads / 32);
    if (grid > want) grid = want;
    const cudaError_t e = launch_overlapped(gen, (unsigned)grid, (unsigned)kAttnGeneralThreads, 0, stream, P);
    if (e != cudaSuccess) return set_cuda_error(e);
    return finish_launch("attn_general");
  }
  int smem = 0;
  const int dp = cache->head_dim <= 64 ? 64 : 128;
  AttnMaps maps;
  memset(&maps, 0, sizeof(maps));
  int rows = kAttnTile;
  while (cache->page_size % rows != 0) rows /= 2;
  if (cache->e4m3 && rows > 32) rows = 32;  // the rows that one warp widens lie together
  P.q_box_tokens = plan.form == kAttnQuad ? 32 / P.group : plan.tok_per_tile;
  bool tma = rows >= 8 && cache->num_pages > 0 && encode_q(&maps.q, P, P.q_box_tokens);
  if (tma) {
    auto both = [&](int kind) {
      P.box_kind = kind;
      // a tile's 128-column rows keep their halves side by side in groups of 8 rows: half a head at a time goes there by eights
      if (kind == kBoxHalf && !cache->e4m3 && dp == 128) rows = 8;
      return encode_side(&maps.k, *cache, P.k, kind, dp, rows) && encode_side(&maps.v, *cache, P.v, kind, dp, rows);
    };
    const int kind = whole_head_kind(*cache);
    tma = both(kind) || (kind != kBoxHalf && both(kBoxHalf));
  }
  if (tma) {
    P.box_rows = rows;
    while ((1 << P.box_shift) < rows) ++P.box_shift;
  }
  AttnTcKernel fn = attn_tc_for(dp, format, plan.form, tma, &smem);
  rc = allow_dynamic_smem((const void*)fn, smem);
  if (rc != QKNORM_OK) return rc;
  rc = attn_tc_registers_ok((const void*)fn);
  if (rc != QKNORM_OK) return rc;
  if (!attn_countable(plan, seqs, cache->heads)) return QKNORM_ERR_SHAPE;
  cudaError_t e = launch_overlapped(fn, (unsigned)plan.grid, (unsigned)kAttnTcThreads, (size_t)smem, stream, P, maps);
  if (e != cudaSuccess) return set_cuda_error(e);
  rc = finish_launch("attn_tc");
  if (rc != QKNORM_OK || !plan.cuts) return rc;
  e = launch_overlapped(attn_join_kernel_for(), dim3((unsigned)plan.grid, (unsigned)(plan.part_rows / kAttnJoinRows)), (unsigned)kAttnJoinThreads, 0, stream, P);
  if (e != cudaSuccess) return set_cuda_error(e);
  return finish_launch("attn_tc");
}

// ---- attention over a 4-bit cache --------------------------------------------------------------------

// How a call over a 4-bit cache is cut: sizes only, so that the workspace can be asked for beforehand.
struct E2m1Plan {
  bool widen = false;
  bool refused = false;  // widen: by "attn_tc", which has to be known before the first launch
  // TMA, where the layout allows it: for whole heads' copies of several heads, and long shares.  us, single tokens of 8 query heads a key
  // head, TMA with 8 (4, 2) heads a copy | cp.async: 64 x 8192 keys 102 | 123, 16 x 32000 keys 97 (102, 106) | 109, 256 x 500 keys 53 | 59, but
  // 64 x 1000 keys 33 | 31, 16 x 2000 keys 27 | 21, 4 x 8192 keys 43 | 23; 2 key heads, 32 x 4000 keys 45 | 32.
  bool tma = false;
  // Eight warps a CTA by cp.async instead of four: where units are no more than SMs, and short enough to be taken whole.  us, eight warps
  // | four: 8 x 1000 keys, 8 key heads of 5 11.4 | 14.8, 16 x 2000 keys, 8 of 8 17.8 | 21.5, 4 x 500 keys 8.3 | 10.3.
  bool wide = false;
  int nt = 1, row_tiles = 1, cols = 0;
  struct Way {  // by cp.async, by TMA
    int heads = 1, grid = 1;
    bool shares = false;
  } way[2];
  int64_t parts = 0;                  // rows of parts, at most
  int64_t side_bytes = 0;             // widened K, or V
  int64_t table_bytes = 0, rest = 0;  // rest: what attn_tc asks for itself
  int64_t cut_bytes = 0;
  int64_t need = 0;
};

// Rows of a sequence and key head from which widening pays: 16 sequences of 4096 keys, 8 key heads, 60 rows 76 us against 112 widened, 95 rows
// 97, 100 rows widened 105; 4 sequences of 8192 keys with 2560 rows 1074 against 252.
constexpr int kE2m1WidenRows = 96;
constexpr int64_t kE2m1WidenMost = (int64_t)2 << 30;    // bytes of the widened cache

E2m1Launch e2m1_kernel(int head_dim, int nt, int copy, bool wide) {
  return head_dim <= 64 ? attn_e2m1_kernel_64(nt, copy, wide) : head_dim <= 128 ? attn_e2m1_kernel_128(nt, copy, wide) : attn_e2m1_kernel_256(nt, copy, wide);
}

// aligned: rows of q and out are, as "attn_tc" wants them.  Rows that are not would be left to the row-at-a-time kernel behind a widened cache.
int plan_e2m1(int seqs, int64_t T, int max_q, int64_t max_keys, int heads_q, int heads_kv, int head_dim, bool causal, int window, bool aligned,
              int sms, E2m1Plan* out) {
  E2m1Plan p;
  const int group = heads_q / heads_kv;
  if ((int64_t)max_q > T) max_q = (int)T;
  const int64_t rows = (int64_t)max_q * group;
  p.cols = (int)((max_keys + kE2m1Page - 1) / kE2m1Page);
  const __int128 wide = (__int128)seqs * p.cols * kE2m1Page * heads_kv * head_dim * 4;  // sizes that a call may have go beyond 64 bits
  const AttnPlan tc = plan_attn(seqs, T, max_q, max_keys, heads_q, heads_kv, head_dim, causal, window, sms);
  p.nt = rows <= 8 ? 1 : 2;
  const int64_t row_tiles = (rows + 8 * p.nt - 1) / (8 * p.nt);
  const bool countable = rows <= 0x7fffffff && row_tiles <= 0x3fffffff / seqs && row_tiles * seqs * heads_kv <= 0x7fffffff;
  if (rows > kE2m1WidenRows && tc.tc && wide <= kE2m1WidenMost && (aligned || !countable)) {
    p.widen = true;
    p.refused = aligned && !attn_countable(tc, seqs, heads_kv);
    p.side_bytes = (int64_t)(wide / 2);
    p.table_bytes = ((int64_t)seqs * p.cols * 4 + 15) / 16 * 16;
    p.rest = attn_workspace(tc, head_dim);
    p.need = 2 * p.side_bytes + p.table_bytes + p.rest + 16;  // 16: the widened cache starts at a multiple of 32 bytes, which its stores take at a time
    *out = p;
    return QKNORM_OK;
  }
  if (!countable) return QKNORM_ERR_SHAPE;
  int64_t span = max_keys;
  if (window > 0) {  // the first row's window, and what the later ones see behind it
    const int64_t w = (int64_t)window + (causal ? max_q : T) - 1;
    if (w < span) span = w;
    span += kE2m1Tile - 1;  // units start at a multiple of a tile
  }
  p.row_tiles = (int)row_tiles;
  const int tma = env_int("QKNORM_E2M1_TMA", -1);  // 0, 1: for tests
  for (int k = 0; k < 2; ++k) {
    if (k == 1 && head_dim != 64 && head_dim != 128) continue;
    E2m1Plan::Way& w = p.way[k];
    if (k == 0) {
      const int wide_round = 8 * kE2m1Tile;
      p.wide = p.nt == 1 && row_tiles * seqs * heads_kv <= sms && (span + wide_round - 1) / wide_round <= kE2m1Whole;
    }
    const E2m1Launch kernel = e2m1_kernel(head_dim, p.nt, k == 1 ? 0 : 16, k == 0 && p.wide);
    while (k == 1 && 2 * w.heads <= kernel.warps && heads_kv % (2 * w.heads) == 0) w.heads *= 2;
    const int round = kE2m1Tile * kernel.warps / w.heads;
    const int64_t places = (int64_t)sms * kernel.per_sm, rounds = (span + round - 1) / round;
    const int64_t units = row_tiles * seqs * (heads_kv / w.heads);
    w.shares = rounds > kE2m1Whole;
    w.grid = (int)(!w.shares || units * rounds < places ? (w.shares ? units * rounds : units) : places);
    if (k == 1) p.tma = tma < 0 ? w.heads >= 4 && units * rounds >= 8 * places : tma != 0;
    if (!w.shares || (k == 1 && !p.tma)) continue;
    const int64_t parts = (int64_t)w.grid * 2 * w.heads * 8 * p.nt;
    if (parts > p.parts) p.parts = parts;
    if (w.grid * 32 > p.cut_bytes) p.cut_bytes = w.grid * 32;
  }
  p.need = p.cut_bytes + (p.parts * (head_dim + 1) * 4 + 15) / 16 * 16;
  *out = p;
  return QKNORM_OK;
}

// One side of a 4-bit cache as [page][head][bytes of a page's tokens], in elements of `element` bytes; a copy takes `run` tokens of
// `heads` heads.  False: no such map.
bool encode_e2m1(CUtensorMap* map, const qknorm_paged_cache_e2m1& c, const AttnSide& s, int token_bytes, int element, int heads, int run) {
  const EncodeTiled enc = encode_tiled();
  if (!enc) return false;
  // the stride of an axis of one is never used, but has to look like one
  const cuuint64_t all = ((cuuint64_t)c.page_size * token_bytes + 15) / 16 * 16;
  const cuuint64_t dims[3] = {(cuuint64_t)c.page_size * token_bytes / element, (cuuint64_t)c.heads, (cuuint64_t)c.num_pages};
  const cuuint64_t strides[2] = {c.heads > 1 ? (cuuint64_t)s.head : all, c.num_pages > 1 ? (cuuint64_t)s.page : all};
  if ((uintptr_t)s.base % 16 != 0) return false;
  for (const cuuint64_t st : strides)
    if (st == 0 || st % 16 != 0 || st >= ((cuuint64_t)1 << 40)) return false;
  const cuuint32_t box[3] = {(cuuint32_t)(run * token_bytes / element), (cuuint32_t)heads, 1};
  const cuuint32_t ones[3] = {1, 1, 1};
  return enc(map, element == 8 ? CU_TENSOR_MAP_DATA_TYPE_INT64 : CU_TENSOR_MAP_DATA_TYPE_INT32, 3, const_cast<void*>(s.base), dims, strides, box, ones,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int check_e2m1_sizes(int32_t seqs, int64_t T, int32_t max_q, int32_t max_kv, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                     int32_t window) {
  const int rc = check_attn_sizes(seqs, T, max_q, max_kv, heads_q, heads_kv, head_dim, window);
  if (rc != QKNORM_OK) return rc;
  return head_dim % 16 != 0 || head_dim > QKNORM_MAX_HEAD_DIM_E2M1 ? QKNORM_ERR_HEADS : QKNORM_OK;
}

int run_attn_e2m1_workspace(int32_t seqs, int64_t T, int32_t max_q, int32_t max_kv, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                            int32_t window, int64_t* bytes) {
  if (!bytes) return QKNORM_ERR_NULL;
  int rc = check_e2m1_sizes(seqs, T, max_q, max_kv, heads_q, heads_kv, head_dim, window);
  if (rc != QKNORM_OK) return rc;
  *bytes = 0;
  if (seqs == 0 || T == 0 || max_q == 0) return QKNORM_OK;
  const DeviceInfo* dev = nullptr;
  rc = current_device(&dev);
  if (rc != QKNORM_OK) return rc;
  for (const bool causal : {true, false})  // enough for either, and wherever q and out lie
    for (const bool aligned : {true, false}) {
      E2m1Plan p;
      rc = plan_e2m1(seqs, T, max_q, max_kv, heads_q, heads_kv, head_dim, causal, window, aligned, dev->sm_count, &p);
      if (rc != QKNORM_OK) return rc;
      if (p.need > *bytes) *bytes = p.need;
    }
  return QKNORM_OK;
}

int run_attn_e2m1(const void* q, int64_t ld_q, const qknorm_paged_cache_e2m1* cache, const int32_t* table, int32_t table_cols,
                  int64_t ld_table, const int32_t* kv_lens, const int32_t* q_starts, int32_t seqs, int64_t T, int32_t max_q, int32_t max_kv,
                  int32_t heads_q, float scale, int32_t causal, int32_t window, void* out, int64_t ld_out, float* lse, void* ws,
                  int64_t ws_bytes, cudaStream_t stream) {
  E2m1Facts f;
  int rc = check_cache(cache, &f);
  if (rc != QKNORM_OK) return rc;
  const int hd = cache->head_dim;
  rc = check_e2m1_sizes(seqs, T, max_q, max_kv, heads_q, cache->heads, hd, window);
  if (rc != QKNORM_OK) return rc;
  if (!(scale > 0.0f) || !isfinite(scale)) return QKNORM_ERR_SHAPE;
  const float c = (float)((double)scale * cache->k_scale * 1.44269504088896340736);
  if (!isfinite(c)) return QKNORM_ERR_SHAPE;
  if (causal != 0 && causal != 1) return QKNORM_ERR_SHAPE;
  if (table_cols < 0 || ld_table < 0 || (ld_table != 0 && ld_table < table_cols)) return QKNORM_ERR_SHAPE;
  AttnE2m1Params E;
  memset(&E, 0, sizeof(E));
  AttnParams& P = E.A;
  const int d = heads_q * hd;
  if ((rc = row_stride(ld_q, d, &P.ld_q)) || (rc = row_stride(ld_out, d, &P.ld_out))) return rc;
  if (seqs == 0 || T == 0 || max_q == 0) return QKNORM_OK;
  if (!q || !out || !kv_lens || !q_starts || (table_cols > 0 && !table)) return QKNORM_ERR_NULL;
  if ((((uintptr_t)q) | ((uintptr_t)out)) & 1u) return QKNORM_ERR_ALIGN;
  if ((((uintptr_t)table) | ((uintptr_t)kv_lens) | ((uintptr_t)q_starts) | ((uintptr_t)lse)) & 3u) return QKNORM_ERR_ALIGN;
  const DeviceInfo* dev = nullptr;
  rc = current_device(&dev);
  if (rc != QKNORM_OK) return rc;
  P.max_keys = (int64_t)table_cols * cache->page_size < max_kv ? (int64_t)table_cols * cache->page_size : max_kv;
  // the plan goes by max_kv, which the workspace was asked for with
  E2m1Plan plan;
  E.q_vec = ((uintptr_t)q | (uintptr_t)P.ld_q * 2) % 16 == 0;
  E.out_vec = ((uintptr_t)out | (uintptr_t)P.ld_out * 2) % 16 == 0;
  rc = plan_e2m1(seqs, T, max_q, max_kv, heads_q, cache->heads, hd, causal != 0, window, E.q_vec && E.out_vec, dev->sm_count, &plan);
  if (rc != QKNORM_OK) return rc;
  if (plan.refused) return QKNORM_ERR_SHAPE;
  const int64_t need = plan.need;
  CallRegions r;
  r.own[r.outs] = -1;
  r.out[r.outs++] = Region{(uintptr_t)out, (uintptr_t)T, (uintptr_t)d * 2, (uintptr_t)P.ld_out * 2};
  if (lse) {
    r.own[r.outs] = -1;
    r.out[r.outs++] = flat(lse, 4 * (uintptr_t)T * heads_q);
  }
  r.in[r.ins++] = Region{(uintptr_t)q, (uintptr_t)T, (uintptr_t)d * 2, (uintptr_t)P.ld_q * 2};
  for (const Region& pool : f.region) r.in[r.ins++] = pool;
  if (table_cols > 0)
    r.in[r.ins++] = Region{(uintptr_t)table, (uintptr_t)seqs, (uintptr_t)table_cols * 4, (uintptr_t)(ld_table ? ld_table : table_cols) * 4};
  r.in[r.ins++] = flat(kv_lens, 4 * (uintptr_t)seqs);
  r.in[r.ins++] = flat(q_starts, 4 * ((uintptr_t)seqs + 1));
  if ((rc = check_regions(r)) != QKNORM_OK) return rc;
  if (need > 0) {
    if (!ws || ws_bytes < need || !aligned16(ws)) return QKNORM_ERR_SCRATCH;
    const Region w = flat(ws, (uintptr_t)need);
    for (int i = 0; i < r.ins; ++i)
      if (may_overlap(w, r.in[i])) return QKNORM_ERR_SCRATCH;
    for (int i = 0; i < r.outs; ++i)
      if (may_overlap(w, r.out[i])) return QKNORM_ERR_SCRATCH;
  }
  P.q = (const uint16_t*)q;
  P.out = (uint16_t*)out;
  P.k = AttnSide{cache->k, cache->k_page, cache->k_token, cache->k_head};
  P.v = AttnSide{cache->v, cache->v_page, cache->v_token, cache->v_head};
  E.ks = AttnSide{cache->k_scales, cache->ks_page, cache->ks_token, cache->ks_head};
  E.vs = AttnSide{cache->v_scales, cache->vs_page, cache->vs_token, cache->vs_head};
  P.num_pages = cache->num_pages;
  P.page_size = cache->page_size;
  P.page_shift = log2_or_minus_one(cache->page_size);
  P.table = table;
  P.ld_table = ld_table ? ld_table : table_cols;
  P.kv_lens = kv_lens;
  P.q_starts = q_starts;
  P.seqs = seqs;
  P.T = T;
  P.max_q = (int64_t)max_q < T ? max_q : (int)T;
  P.heads_q = heads_q;
  P.heads_kv = cache->heads;
  P.group = heads_q / cache->heads;
  P.head_dim = hd;
  P.c = c;
  P.v_scale = cache->v_scale;
  P.causal = causal;
  P.window = window;
  P.lse = lse;
  P.error = dev->ring_error;

  if (plan.widen) {
    WidenParams W;
    W.P = E;
    W.k = (uint16_t*)(((uintptr_t)ws + 31) & ~(uintptr_t)31);
    W.v = (uint16_t*)((char*)W.k + plan.side_bytes);
    W.table = (int*)((char*)W.k + 2 * plan.side_bytes);
    W.cols = plan.cols;
    const int64_t ctas = (int64_t)seqs * plan.cols * cache->heads;
    if (ctas > 0) {
      const cudaError_t e = launch_overlapped(e2m1_widen_kernel_for(), (unsigned)ctas, (unsigned)kE2m1WidenThreads, 0, stream, W);
      if (e != cudaSuccess) return set_cuda_error(e);
      rc = finish_launch("attn_e2m1");
      if (rc != QKNORM_OK) return rc;
    }
    qknorm_paged_cache wide = {};
    wide.k = W.k;
    wide.v = W.v;
    wide.k_token = wide.v_token = hd;
    wide.k_head = wide.v_head = (int64_t)kE2m1Page * hd;
    wide.k_page = wide.v_page = (int64_t)cache->heads * kE2m1Page * hd;
    wide.num_pages = (int64_t)seqs * plan.cols;
    wide.page_size = kE2m1Page;
    wide.heads = cache->heads;
    wide.head_dim = hd;
    const float s = fmaxf((float)((double)scale * cache->k_scale), 1.401298464e-45f);
    return run_attn(q, ld_q, &wide, W.table, plan.cols, 0, kv_lens, q_starts, seqs, T, max_q, (int)P.max_keys, heads_q, s, causal, window,
                    out, ld_out, lse, (char*)W.table + plan.table_bytes, plan.rest, stream, true, cache->v_scale);
  }

  if (cache->num_pages == 0) {  // never read, but copies of no bytes name an address, too, and one that their size divides
    const AttnSide none = {(const void*)((uintptr_t)q & ~(uintptr_t)15), 0, 0, 0};
    P.k = P.v = E.ks = E.vs = none;
  }
  E.row_tiles = plan.row_tiles;
  E.tile_rows = 8 * plan.nt;
  const int blocks = hd / 16, low = blocks & -blocks;
  E.scale_unit = low > 8 ? 8 : low;
  if (plan.parts > 0) {
    E.cuts = (int*)ws;
    E.part_o = (float*)((char*)ws + plan.cut_bytes);
    E.part_z = E.part_o + plan.parts * hd;
  }
  E2m1Maps maps;
  memset(&maps, 0, sizeof(maps));
  int copy = f.vec16 ? 16 : 8;
  // TMA: tokens of a head one after the other in codes and scales, everything on 16 bytes, pages of whole runs of 16 tokens; copies go to
  // multiples of 128 bytes.
  const int heads = plan.way[1].heads;
  E.run_shift = cache->page_size % 32 == 0 ? 5 : 4;
  if ((hd == 64 || hd == 128) && cache->page_size % 16 == 0 && cache->num_pages > 0 && P.k.token == hd / 2 && P.v.token == hd / 2 &&
      E.ks.token == hd / 16 && E.vs.token == hd / 16 && (heads << E.run_shift) * (hd / 16) % 128 == 0 && plan.tma &&
      encode_e2m1(&maps.k, *cache, P.k, hd / 2, 8, heads, 1 << E.run_shift) && encode_e2m1(&maps.v, *cache, P.v, hd / 2, 8, heads, 1 << E.run_shift) &&
      encode_e2m1(&maps.ks, *cache, E.ks, hd / 16, 4, heads, 1 << E.run_shift) &&
      encode_e2m1(&maps.vs, *cache, E.vs, hd / 16, 4, heads, 1 << E.run_shift))
    copy = 0;
  const E2m1Plan::Way& way = plan.way[copy == 0];
  E.heads_cta = way.heads;
  E.shares = way.shares;
  P.grid = way.grid;
  const E2m1Launch kernel = e2m1_kernel(hd, plan.nt, copy, copy != 0 && plan.wide);
  rc = allow_dynamic_smem((const void*)kernel.fn, kernel.smem);
  if (rc != QKNORM_OK) return rc;
  cudaError_t e = launch_overlapped(kernel.fn, (unsigned)way.grid, (unsigned)(32 * kernel.warps), (size_t)kernel.smem, stream, E, maps);
  if (e != cudaSuccess) return set_cuda_error(e);
  rc = finish_launch("attn_e2m1");
  if (rc != QKNORM_OK || !way.shares) return rc;
  e = launch_overlapped(attn_e2m1_join_kernel_for(), dim3((unsigned)way.grid, (unsigned)((way.heads * 8 * plan.nt + 7) / 8)),
                        (unsigned)kE2m1JoinThreads, 0, stream, E);
  if (e != cudaSuccess) return set_cuda_error(e);
  return finish_launch("attn_e2m1");
}
