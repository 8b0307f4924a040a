// The kernels of wkv_decode.hip that also accumulate attention weights; a file of their own, so that both compile side by side.
#define WKV_DECODE_WEIGHTED
#include "wkv_decode.hip"
