/* launch_recorder.c, and the lanes of a launch along each dimension of its grid. */
#include "launch_recorder.c"

uint64_t recorder_lanes(int i, int dim) {
  const launch_t *l = &launches[i];
  return dim == 0 ? (uint64_t)l->grid.x * l->block.x : dim == 1 ? (uint64_t)l->grid.y * l->block.y : (uint64_t)l->grid.z * l->block.z;
}
uint64_t recorder_grid(int i, int dim) { return dim == 0 ? launches[i].grid.x : dim == 1 ? launches[i].grid.y : launches[i].grid.z; }
