// C entry points of the hosted-model operators: argument checks on the host, then the launchers.
#include "hosted.cuh"

namespace approxifer {
namespace {

constexpr int64_t kMaxExtent = 0x7fffffffLL;

bool whole(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
int type_bytes(int32_t type) { return type == APPROXIFER_TYPE_F32 ? 4 : 2; }
bool known_type(int32_t type) { return type == APPROXIFER_TYPE_BF16 || type == APPROXIFER_TYPE_F32; }
int from_cuda(cudaError_t e) { return e == cudaSuccess ? APPROXIFER_OK : APPROXIFER_E_CUDA; }

}  // namespace

namespace {
// Everything but the pointers.
int check_attention(const approxifer_attention_args& a) {
  if (a.T < 0 || a.T > kMaxExtent || a.batch < 0 || a.max_q < 0 || a.Hq < 1 || a.Hq > 65535 || a.Hkv < 1 || a.D < 1 || a.D > 256) return APPROXIFER_E_RANGE;
  if (a.page_size < 1 || a.window < 0 || a.sinks < 0 || a.num_pages < 0 || a.num_pages > kMaxExtent || a.table_pages < 0 || a.table_pages > kMaxExtent ||
      a.workspace_bytes < 0)
    return APPROXIFER_E_RANGE;
  if (a.q_tstride < 0 || a.q_hstride < a.D || a.o_tstride < 0 || a.o_hstride < a.D || a.kc_rstride < a.D || a.kc_hstride < a.D || a.kc_pstride < a.D ||
      a.vc_rstride < a.D || a.vc_hstride < a.D || a.vc_pstride < a.D || a.table_stride < 0)
    return APPROXIFER_E_RANGE;
  if (a.Hq % a.Hkv != 0 || a.reserved != 0 || !isfinite(a.scale)) return APPROXIFER_E_PARAM;
  if (a.T > (int64_t)a.batch * a.max_q) return APPROXIFER_E_RANGE;  // (some sequence has more queries than max_q: their rows would not be written)
  return APPROXIFER_OK;
}
}  // namespace

cudaError_t read_hosted_wait_timeouts(unsigned int* out) {
  *out = 0;
  for (auto read : {read_linear_tile_wait_timeouts, read_linear_pair_wait_timeouts, read_attention_tile_wait_timeouts}) {
    unsigned int n = 0;
    const cudaError_t e = read(&n);
    if (e != cudaSuccess) return e;
    *out += n;
  }
  return cudaSuccess;
}
cudaError_t reset_hosted_wait_timeouts() {
  for (auto reset : {reset_linear_tile_wait_timeouts, reset_linear_pair_wait_timeouts, reset_attention_tile_wait_timeouts}) {
    const cudaError_t e = reset();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace approxifer

using namespace approxifer;

extern "C" {

int approxifer_linear(const approxifer_linear_args* a, void* cuda_stream) {
  if (a == nullptr) return APPROXIFER_E_NULL;
  if (a->M < 0 || a->M > kMaxExtent || a->N < 1 || a->N > kMaxExtent || a->K < 1 || a->K > kMaxExtent) return APPROXIFER_E_RANGE;
  if (a->x_rstride < a->K || a->w_rstride < a->K || a->y_rstride < a->N || (a->R && a->r_rstride < a->N)) return APPROXIFER_E_RANGE;
  if (a->activation < APPROXIFER_ACT_NONE || a->activation > APPROXIFER_ACT_SILU || !known_type(a->out_type)) return APPROXIFER_E_PARAM;
  if (a->M == 0) return APPROXIFER_OK;
  if (!a->X || !a->Wt || !a->Y) return APPROXIFER_E_NULL;
  const int size = type_bytes(a->out_type);
  if (!whole(a->X, 2) || !whole(a->Wt, 2) || !whole(a->bias, 2) || !whole(a->R, size) || !whole(a->Y, size)) return APPROXIFER_E_PARAM;
  return from_cuda(launch_linear(*a, static_cast<cudaStream_t>(cuda_stream)));
}

int approxifer_qk_norm_rope(const approxifer_norm_rope_args* a, void* cuda_stream) {
  if (a == nullptr) return APPROXIFER_E_NULL;
  if (a->T < 0 || a->T > kMaxExtent || a->Hq < 1 || a->Hq > 65535 || a->Hkv < 1 || a->Hkv > 65535 || a->D < 1 || a->D > 256) return APPROXIFER_E_RANGE;
  if (a->rot < 0 || a->rot > a->D || a->page_size < 1 || a->num_pages < 0 || a->num_pages > kMaxExtent || a->positions_max < 0) return APPROXIFER_E_RANGE;
  if (a->rot % 2 != 0 || !known_type(a->type) || !(a->eps >= 0.f)) return APPROXIFER_E_PARAM;
  if ((a->k == nullptr) != (a->k_cache == nullptr) || (a->v == nullptr) != (a->v_cache == nullptr)) return APPROXIFER_E_NULL;
  if (a->q_tstride < 0 || a->q_hstride < a->D || a->qo_tstride < 0 || a->qo_hstride < a->D) return APPROXIFER_E_RANGE;
  if (a->k && (a->k_tstride < 0 || a->k_hstride < a->D || a->kc_rstride < a->D || a->kc_hstride < a->D || a->kc_pstride < a->D)) return APPROXIFER_E_RANGE;
  if (a->v && (a->v_tstride < 0 || a->v_hstride < a->D || a->vc_rstride < a->D || a->vc_hstride < a->D || a->vc_pstride < a->D)) return APPROXIFER_E_RANGE;
  if (a->T == 0) return APPROXIFER_OK;
  if (!a->q || !a->q_out || (a->rot && (!a->cos_sin || !a->positions)) || ((a->k || a->v) && !a->slots)) return APPROXIFER_E_NULL;
  const int size = type_bytes(a->type);
  if (!whole(a->q, size) || !whole(a->k, size) || !whole(a->v, size) || !whole(a->q_out, size) || !whole(a->k_cache, size) ||
      !whole(a->v_cache, size) || !whole(a->q_weight, size) || !whole(a->k_weight, size) || !whole(a->cos_sin, 4))
    return APPROXIFER_E_PARAM;
  return from_cuda(launch_norm_rope(*a, static_cast<cudaStream_t>(cuda_stream)));
}

int64_t approxifer_attention_workspace(const approxifer_attention_args* a) {
  if (a == nullptr) return APPROXIFER_E_NULL;
  const int rc = check_attention(*a);
  if (rc) return rc;
  return a->T > 0 && attention_token_eligible(*a) ? attention_token_workspace(*a) : 0;
}

int approxifer_attention(const approxifer_attention_args* a, void* cuda_stream) {
  if (a == nullptr) return APPROXIFER_E_NULL;
  const int rc = check_attention(*a);
  if (rc) return rc;
  if (a->T == 0) return APPROXIFER_OK;
  if (!a->q || !a->k_cache || !a->v_cache || !a->q_start || !a->kv_len || !a->out || (a->table_pages > 0 && !a->block_table)) return APPROXIFER_E_NULL;
  if (!whole(a->q, 2) || !whole(a->k_cache, 2) || !whole(a->v_cache, 2) || !whole(a->out, 2) || !whole(a->workspace, 16)) return APPROXIFER_E_PARAM;
  return from_cuda(launch_attention(*a, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
