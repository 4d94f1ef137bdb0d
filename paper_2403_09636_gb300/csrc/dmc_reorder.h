// Limits of a reordering call. Host and device.
#pragma once

namespace dmc {

constexpr int kReorderRows = 512;  // sequences of one call

}  // namespace dmc
