// What the translation units of the library share on the host side.
#pragma once
#include <cstdint>

namespace wm {

constexpr uint32_t kInjectNoScanner = 1u, kInjectNoCopy = 2u, kInjectNoMeasures = 4u;    // wm_inject_stall

extern thread_local uint32_t g_launches;      // kernels the last call on this thread enqueued
uint32_t wait_budget_ns();                    // wm_wait_budget_ms
uint32_t inject_bits();

}  // namespace wm
