// Stands before the HIP runtime in a process without a GPU: launches are noted, not made, and succeed, so that the host side of an entry point can be looked at
// with addresses that nobody follows.  (Preloaded: tests/test_launch_sizes.py.)
typedef struct {
  unsigned x, y, z;
} dim;
#define MOST 4096
static dim grids[MOST], blocks[MOST];
static int count;
// a launch is made of three calls: its sizes are put down, taken up again by the kernel's stub, and passed on
static dim grid_now, block_now;
int __hipPushCallConfiguration(dim grid, dim block, unsigned long shared, void* stream) {
  (void)shared, (void)stream;
  grid_now = grid, block_now = block;
  return 0;
}
int __hipPopCallConfiguration(dim* grid, dim* block, unsigned long* shared, void** stream) {
  *grid = grid_now, *block = block_now, *shared = 0, *stream = 0;
  return 0;
}
int hipLaunchKernel(const void* f, dim grid, dim block, void** args, unsigned long shared, void* stream) {
  (void)f, (void)args, (void)shared, (void)stream;
  if (count < MOST) grids[count] = grid, blocks[count] = block;
  ++count;
  return 0;
}
int hipGetLastError(void) { return 0; }
int launches(void) { return count; }
void forget(void) { count = 0; }
void launch(int i, unsigned* out) {
  out[0] = grids[i].x, out[1] = grids[i].y, out[2] = grids[i].z, out[3] = blocks[i].x, out[4] = blocks[i].y, out[5] = blocks[i].z;
}
