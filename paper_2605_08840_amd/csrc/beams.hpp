// Beams over a paged cache: what its kernels share.
#pragma once

#include "pages.hpp"

namespace restkv {

struct Beams {
  int n_groups, n_beams, n_vocab, n_out, dtype, end_token;
  int64_t stride;
};
int resolve_beams(const restkv_beams* b, Beams* o);

size_t beam_ws_bytes(const Beams& b);
int launch_beam_select(const Beams& b, const void* logits, const float* scores, const int32_t* finished, float* new_scores,
                       int32_t* parents, int32_t* tokens, int32_t* new_finished, char* ws, hipStream_t st);
int launch_beam_reorder(const Pages& pg, int n_beams, const int32_t* parents, int64_t parents_stride, int32_t* table_out,
                        const restkv_layer_pages* layers, int n_layers, hipStream_t st);
void force_shared(bool on);     // see restkv_debug_force_shared
int beams_list(const Pages& pg, int n_beams, const int32_t* tiles, int32_t* chunks);       // see restkv_debug_beams_list
size_t attend_beams_ws_bytes(const Pages& pg, int n_beams);
int launch_attend_beams(const Pages& pg, int n_beams, const int32_t* shared, const void* q, const void* k_pages, const void* v_pages,
                        const void* k_scale, const void* v_scale, void* out, float* lse, char* ws, hipStream_t st);

}  // namespace restkv
