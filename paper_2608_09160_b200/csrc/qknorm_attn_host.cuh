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

struct CallRegions {  // buffers of a call: outputs, and everything an output must not touch
  Region out[8], in[16];
  int outs = 0, ins = 0;
  int own[8];            // out[i] may be exactly in[own[i]]
  int pools = -1;        // out[pools] and out[pools + 1] are the two sides of a cache, looked at apart from the others
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
      if (j != i && !(c.pools >= 0 && i + j == 2 * c.pools + 1 && (i == c.pools || j == c.pools)) && may_overlap(c.out[i], c.out[j]))
        return QKNORM_ERR_ALIAS;
  }
  return QKNORM_OK;
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

int run_rope(int elem_bytes, const void* q, const void* k, const qknorm_rotation* rot, int64_t T, int32_t dq, int32_t dk,
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
  if ((rc = check_rotation(rot, head_dim, R)) != QKNORM_OK) return rc;
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
  if (R.rot_dim) {
    c.in[c.ins++] = flat(R.positions, 8 * (uintptr_t)T);
    c.in[c.ins++] = flat(R.inv_freq, 4 * (uintptr_t)R.rot_dim);
  }
  if ((rc = check_regions(c)) != QKNORM_OK) return rc;
  return launch_rope(R, elem_bytes, 0, kNormNone, aligned, stream);
}

int run_append(const void* q, const void* k, const void* v, const void* gq, const void* gk, int32_t norm, float eps,
               const qknorm_rotation* rot, const int64_t* slots, const qknorm_paged_cache* cache, int64_t T, int32_t dq, int64_t ld_q,
               int64_t ld_k, int64_t ld_v, void* oq, int64_t ld_oq, cudaStream_t stream) {
  CacheFacts f;
  int rc = check_cache(cache, &f);
  if (rc != QKNORM_OK) return rc;
  const int hd = cache->head_dim, dk = cache->heads * hd;
  if (T < 0 || dq < 0 || dq > kMaxDim) return QKNORM_ERR_SHAPE;
  if (dq % hd != 0) return QKNORM_ERR_HEADS;
  if (norm < kNormNone || norm > kNormHead) return QKNORM_ERR_SHAPE;
  if (norm != kNormNone && !(eps >= 0.0f)) return QKNORM_ERR_EPS;
  if (cache->e4m3 && (!isfinite(1.0f / cache->k_scale) || !isfinite(1.0f / cache->v_scale))) return QKNORM_ERR_SHAPE;
  RopeParams R;
  memset(&R, 0, sizeof(R));
  if ((rc = row_stride(ld_q, dq, &R.q.ldx)) || (rc = row_stride(ld_oq, dq, &R.q.ldy)) || (rc = row_stride(ld_k, dk, &R.k.ldx)) ||
      (rc = row_stride(ld_v, dk, &R.v.ldx)))
    return rc;
  if (T == 0) return QKNORM_OK;
  if ((rc = check_rotation(rot, hd, R)) != QKNORM_OK) return rc;
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
  R.ck = CacheSide{cache->k, cache->k_page, cache->k_token, cache->k_head, cache->e4m3 ? 1.0f / cache->k_scale : 1.0f};
  R.cv = CacheSide{cache->v, cache->v_page, cache->v_token, cache->v_head, cache->e4m3 ? 1.0f / cache->v_scale : 1.0f};
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
  c.own[c.outs] = -1;
  c.out[c.outs++] = f.k;
  c.own[c.outs] = -1;
  c.out[c.outs++] = f.v;
  c.in[c.ins++] = Region{(uintptr_t)k, rows, kb, (uintptr_t)R.k.ldx * 2};
  c.in[c.ins++] = Region{(uintptr_t)v, rows, kb, (uintptr_t)R.v.ldx * 2};
  if (norm != kNormNone) c.in[c.ins++] = flat(gk, kb);
  c.in[c.ins++] = flat(slots, 8 * rows);
  if (R.rot_dim) {
    c.in[c.ins++] = flat(R.positions, 8 * rows);
    c.in[c.ins++] = flat(R.inv_freq, 4 * (uintptr_t)R.rot_dim);
  }
  if ((rc = check_regions(c)) != QKNORM_OK) return rc;
  if (cache->num_pages > 0 && pools_meet(pool_shape(*cache, cache->k, cache->k_page, cache->k_token, cache->k_head),
                                         pool_shape(*cache, cache->v, cache->v_page, cache->v_token, cache->v_head)))
    return QKNORM_ERR_ALIAS;
  const bool vec = (hd | R.rot_dim) % 16 == 0 && ptrs % 16 == 0 && strides % 8 == 0 && (cache->e4m3 ? f.vec8 : f.vec16);
  return launch_rope(R, 2, cache->e4m3 ? 1 : 2, norm, vec, stream);
}

// ---- attention over the paged cache ---------------------------------------------------------------

AttnTcKernel attn_tc_for(int dp, bool e4m3, int form, bool tma, int* smem) {
  if (dp == 64) return e4m3 ? attn_tc_kernel_e4m364(form, tma, smem) : attn_tc_kernel_bf1664(form, tma, smem);
  return e4m3 ? attn_tc_kernel_e4m3128(form, tma, smem) : attn_tc_kernel_bf16128(form, tma, smem);
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

int run_attn(const void* q, int64_t ld_q, const qknorm_paged_cache* cache, const int32_t* table, int32_t table_cols, int64_t ld_table,
             const int32_t* kv_lens, const int32_t* q_starts, int32_t seqs, int64_t T, int32_t max_q, int32_t max_kv, int32_t heads_q,
             float scale, int32_t causal, int32_t window, void* out, int64_t ld_out, float* lse, void* ws, int64_t ws_bytes,
             cudaStream_t stream) {
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
  P.v_scale = cache->e4m3 ? cache->v_scale : 1.0f;
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
    AttnKernel gen = attn_general_kernel_for(cache->e4m3 != 0);
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
  AttnTcKernel fn = attn_tc_for(dp, cache->e4m3 != 0, plan.form, tma, &smem);
  rc = allow_dynamic_smem((const void*)fn, smem);
  if (rc != QKNORM_OK) return rc;
  rc = attn_tc_registers_ok((const void*)fn);
  if (rc != QKNORM_OK) return rc;
  if ((int64_t)plan.q_items * seqs > 0x3fffffff || (int64_t)seqs * cache->heads > 0x3fffffff) return QKNORM_ERR_SHAPE;
  cudaError_t e = launch_overlapped(fn, (unsigned)plan.grid, (unsigned)kAttnTcThreads, (size_t)smem, stream, P, maps);
  if (e != cudaSuccess) return set_cuda_error(e);
  rc = finish_launch("attn_tc");
  if (rc != QKNORM_OK || !plan.cuts) return rc;
  e = launch_overlapped(attn_join_kernel_for(), dim3((unsigned)plan.grid, (unsigned)(plan.part_rows / kAttnJoinRows)), (unsigned)kAttnJoinThreads, 0, stream, P);
  if (e != cudaSuccess) return set_cuda_error(e);
  return finish_launch("attn_tc");
}
