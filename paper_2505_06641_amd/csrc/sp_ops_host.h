// What the C entry points of the operators (sp_ops*.hip) share on the host: the handle, checks of addresses, teams for rows.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "sneakpeek.h"
#include "sp_host.h"
#include "sp_ops_common.h"

struct sp_ops {
  int device = 0;
  char* ws = nullptr;              // partial sums
  int64_t ws_bytes = 0;
  uint32_t* err = nullptr;         // behind them: kErr* bits since the last sp_ops_check; those of the last one
  std::string hip_err;
};

namespace sp {

inline bool dtype_ok(int32_t t) { return t == SP_F32 || t == SP_BF16; }
inline int64_t elem_bytes(int32_t t) { return t == SP_F32 ? 4 : 2; }
// Elements at their own size's multiples; null passes.
inline bool aligned(const void* p, int32_t t) { return ((uintptr_t)p & (uintptr_t)(elem_bytes(t) - 1)) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

inline sp_status launched(sp_ops* o) {
  SP_HIP(o, hipGetLastError());
  return SP_OK;
}

// Calls f<TEAM, C>() with the smallest team that holds rows of `pieces` 16-byte pieces: parts of a wavefront for narrow rows, so
// that no lane idles, one wavefront with up to four pieces a lane (a sum over lanes costs a wavefront nothing but its own
// instructions, one over a workgroup two barriers), then workgroups.  False where no team does.
template <typename F>
bool with_team(int64_t pieces, F&& f) {
  if (pieces <= 2) f.template operator()<2, 1>();
  else if (pieces <= 4) f.template operator()<4, 1>();
  else if (pieces <= 8) f.template operator()<8, 1>();
  else if (pieces <= 16) f.template operator()<16, 1>();
  else if (pieces <= 32) f.template operator()<32, 1>();
  else if (pieces <= 64) f.template operator()<64, 1>();
  else if (pieces <= 128) f.template operator()<64, 2>();
  else if (pieces <= 256) f.template operator()<64, 4>();
  else if (pieces <= 512) f.template operator()<256, 2>();
  else if (pieces <= 1024) f.template operator()<256, 4>();
  else if (pieces <= 2048) f.template operator()<1024, 2>();
  else if (pieces <= 4096) f.template operator()<1024, 4>();
  else return false;
  return true;
}

}  // namespace sp
