// The host side of the library with a look at the launch geometry that uniprefill_attention takes.
#include "up_api.hip"

// out: rows of a work-group, keys of a piece (0: the keys are not cut)
extern "C" int attn_form(const up_params* p, const int32_t* cu, const int32_t* cu_k, int32_t* out) {
  Problem pb;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  AttnGeometry g;
  if ((st = attn_geometry(pb, cu, cu_k, &g)) != UP_OK) return st;
  out[0] = g.rows;
  out[1] = g.part_keys;
  return UP_OK;
}
