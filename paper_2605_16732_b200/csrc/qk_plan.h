// What the kernels behind a dirotq_qk_t take from it, in one place for all entry points.  Plain C++.
#pragma once
#include "../../include/dirotq.h"

namespace dirotq {

// The tokens' positions, or NULL where a token's row is its position.  Where nothing is rotated the description's pointer is not looked at: it
// need not hold M positions then, nor point anywhere (qk_check leaves it unchecked too).
inline const int32_t* qk_positions(const dirotq_qk_t& qk) { return qk.rope != DIROTQ_ROPE_NONE ? qk.positions : nullptr; }

}  // namespace dirotq
