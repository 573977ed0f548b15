// Grids of more workgroups than one dimension holds: a grid dimension has fewer than 2^32
// threads, so workgroup L of n is (L % x, L / x) of rows of x = 2^16 workgroups; those from n
// on end at once. Plain C so that a host test can check that.
#ifndef QWM_GRID_ROWS_H
#define QWM_GRID_ROWS_H

#include <stdint.h>

static inline uint32_t qwm_grid_x(int64_t n) { return n < 65536 ? (uint32_t)n : 65536u; }
static inline uint32_t qwm_grid_y(int64_t n) { return (uint32_t)((n + 65535) / 65536); }

#endif
