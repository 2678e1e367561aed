// The stage calls with their arguments in one struct (include/agora_stage.h).  The caller's layer takes about 0.1 us for an argument
// of a C call; one block of bytes takes 0.6 us for any number of them.
#include "agora_stage.h"

extern "C" {

ssn_status_t stage_qk_rope_forward_packed(const stage_qk_rope_forward_args_t *a) {
  if (a == nullptr) return SSN_ERR_NULL;
  return stage_qk_rope_forward(a->op, a->q, a->q_token, a->q_head, a->q_heads, a->k, a->k_token, a->k_head, a->k_heads, a->q_out, a->qo_token,
                               a->qo_head, a->k_out, a->ko_token, a->ko_head, a->pos, a->n_tokens, a->seq_len, a->stream);
}

ssn_status_t stage_qk_rope_backward_packed(const stage_qk_rope_backward_args_t *a) {
  if (a == nullptr) return SSN_ERR_NULL;
  return stage_qk_rope_backward(a->op, a->dq, a->dq_token, a->dq_head, a->dk, a->dk_token, a->dk_head, a->q, a->q_token, a->q_head, a->q_heads,
                                a->k, a->k_token, a->k_head, a->k_heads, a->dq_in, a->dqi_token, a->dqi_head, a->dk_in, a->dki_token,
                                a->dki_head, a->dwq, a->dwk, a->pos, a->n_tokens, a->seq_len, a->workspace, a->workspace_bytes, a->stream);
}

ssn_status_t stage_distill_loss_packed(const stage_distill_loss_args_t *a) {
  if (a == nullptr) return SSN_ERR_NULL;
  return stage_distill_loss(a->logits, a->ldl, a->dtype, a->n_tokens, a->vocab, a->ids, a->ldi, a->top, a->ldt, a->top_k, a->weight, a->tau,
                            a->loss, a->dlogits, a->ldd, a->dev_status, a->stream);
}

ssn_status_t stage_int8_quantize_packed(const stage_int8_quantize_args_t *a) {
  if (a == nullptr) return SSN_ERR_NULL;
  return stage_int8_quantize(a->x, a->ldx, a->dtype, a->rows, a->cols, a->q, a->ldq, a->scale, a->stream);
}

ssn_status_t stage_int8_matmul_packed(const stage_int8_matmul_args_t *a) {
  if (a == nullptr) return SSN_ERR_NULL;
  return stage_int8_matmul(a->xq, a->ldx, a->xs, a->wq, a->ldw, a->ws, a->n_tokens, a->inner, a->outer, a->y, a->ldy, a->dtype, a->dev_status,
                           a->stream);
}

}  // extern "C"
