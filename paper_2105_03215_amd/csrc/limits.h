// Limits that the schema's checks and the kernels share.
#pragma once

namespace byoc {

constexpr int kMaxTree = 256;  // drafted tokens of a sequence, whose paths the kernels hold as bits in LDS

}  // namespace byoc
