/* fake_hip.c, with every launch's grid, workgroup and the beginning of its first argument kept besides its name.  Preloaded by
 * tests/test_gated_launches.py.  Test infrastructure only. */
#define __hipPushCallConfiguration listed_push
#define __hipPopCallConfiguration listed_pop
#define hipLaunchKernel listed_launch
#include "fake_hip.c"
#undef __hipPushCallConfiguration
#undef __hipPopCallConfiguration
#undef hipLaunchKernel

struct size3 { unsigned x, y, z; };
struct kept { unsigned grid, threads; unsigned char argument[128]; };
static struct size3 grid_, block_;
static struct kept kept[256];
static int n_kept;

int fake_kept(struct kept *to) { int n = n_kept; memcpy(to, kept, sizeof kept); n_kept = 0; return n; }

int __hipPushCallConfiguration(struct size3 grid, struct size3 block, size_t shared, void *stream)
{
    (void)shared; (void)stream;
    grid_ = grid; block_ = block;
    return OK;
}
int __hipPopCallConfiguration(struct size3 *grid, struct size3 *block, size_t *shared, void **stream)
{
    *grid = grid_; *block = block_; *shared = 0; *stream = NULL;
    return OK;
}
int hipLaunchKernel(const void *host, struct size3 grid, struct size3 block, void **arguments)
{
    if (n_kept < 256) {
        kept[n_kept].grid = grid.x; kept[n_kept].threads = block.x;
        memcpy(kept[n_kept++].argument, arguments[0], sizeof kept[0].argument);
    }
    return listed_launch(host);
}
