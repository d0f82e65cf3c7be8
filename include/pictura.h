/*
 * pictura.h -- C ABI of the MI355X (gfx950) batched class/depth view rasterizer.
 *
 * The library renders, for every agent of every world and every camera of
 * the agent's rig, a perspective image of the surrounding agents' boxes and
 * the static map triangles (paper Sec. 3.2, Eq. obs_pv: I_ik = Phi(A_i, W_i,
 * K_ik); "only the surroundings are rendered", so a view never draws its own
 * agent).  Each pixel receives the class ID of the nearest surface (uint8)
 * and its view-space depth in metres (fp32, +inf for background).  Fixed
 * rules make the result independent of triangle order and of how the work is
 * split (all fp32 arithmetic without contraction, correctly rounded
 * divisions): R1 camera = agent pose composed with the mount (yaw only);
 * R2 view transform; R3 1/z plane of the unsnapped triangle; R4 Sutherland-
 * Hodgman clip against z = near, fanned from the first vertex, and a
 * triangle whose three vertices all lie beyond far (or all nearer than near)
 * is not drawn, since no point of it lies inside the view volume; R5 snap to
 * 1/256 pixel, ties to even; R6 exact integer edge functions at pixel
 * centres, top-left fill rule, two-sided; R7 key = (24-bit reverse depth from
 * the fp32 bits of 1/z, capped at the power of two above 1/near) << 8 | class,
 * the minimum key wins, 1/z below 1/far is rejected; R8 depth = 1 / the code's
 * bucket midpoint; R9 agent boxes of 12 triangles, the ego's own box skipped.
 *
 * Conventions
 *  - Plain C99; no HIP/CUDA or C++ types.  A `void* stream` is a hipStream_t
 *    (NULL = the device's null stream).  Device pointers are HIP device
 *    allocations on the context's device; host pointers are ordinary memory.
 *  - Every call returns a pictura_status.  Argument errors are detected on the
 *    host and returned synchronously without launching anything; the context
 *    stays usable after any error.  pictura_last_error() gives a message.
 *  - Work is enqueued on `stream` and the calls return without synchronising,
 *    except where a call says that it waits or copies to host memory.
 *  - A context is not thread-safe: use one context per host thread.
 *  - Render kernels read the agents' arrays in place.  A render call on another
 *    stream than the previous render call of the context is ordered after that
 *    call's kernels (an event wait on the device, not a host synchronisation).
 */
#ifndef PICTURA_H
#define PICTURA_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t pictura_status;
#define PICTURA_OK        0
#define PICTURA_EINVAL   (-1) /* bad argument (null pointer, size, rig value) */
#define PICTURA_ENOMEM   (-2) /* device allocation failed */
#define PICTURA_EDEVICE  (-3) /* no usable HIP device, or a HIP call failed */
#define PICTURA_ESTATE   (-4) /* call order violated (e.g. render before binning) */
#define PICTURA_ERANGE   (-5) /* a size exceeds a supported limit */

#define PICTURA_MAX_CAMS 8

typedef struct pictura_ctx_s* pictura_ctx;

/* Static scene of all worlds (host memory; the library copies it).
 * Triangles are concatenated world by world: world w owns triangles
 * [tri_offsets[w], tri_offsets[w+1]).  verts[t] = x0 y0 z0 x1 y1 z1 x2 y2 z2 in
 * world metres (z up).  cls[t] is the class ID (0..254).  bounds[w] =
 * xmin ymin xmax ymax is the rectangle the world's binning grid covers;
 * triangles outside it are still drawn (they are binned into edge cells). */
typedef struct {
    int32_t num_worlds;
    const int64_t* tri_offsets; /* host, [num_worlds + 1], non-decreasing, [0] == 0 */
    const float* verts;         /* host, [T][9] */
    const uint8_t* cls;         /* host, [T] */
    const float* bounds;        /* host, [num_worlds][4] */
} pictura_scene;

/* Agents (device memory, caller-owned, structure of arrays).  Agent
 * g = w * agents_per_world + a; (cos_h, sin_h) is its heading; the box spans
 * length x width around (x, y) and z0 .. z0 + height. */
typedef struct {
    int32_t num_worlds;
    int32_t agents_per_world;
    const float* x;
    const float* y;
    const float* z0;
    const float* cos_h;
    const float* sin_h;
    const float* length;
    const float* width;
    const float* height;
    const uint8_t* cls;
} pictura_agents;

/* Camera rig shared by all agents (host, by value).  Pinhole intrinsics in
 * pixels (x right, y down, pixel (i, j) centre at (i + 0.5, j + 0.5)); mount k
 * = x y z cos_yaw sin_yaw in the ego frame (x forward, y left, z up; paper
 * App. A.2, Tab. camera_rig).  near_m > 0, far_m > near_m. */
typedef struct {
    int32_t num_cams;
    int32_t width;
    int32_t height;
    float fx, fy, cx, cy;
    float near_m, far_m;
    float mount[PICTURA_MAX_CAMS][5];
} pictura_rig;

/* Mutable kinematic-bicycle state (device memory, caller-owned). */
typedef struct {
    int32_t count;
    float* x;
    float* y;
    float* psi;      /* heading angle, kept in (-pi, pi] */
    float* speed;    /* m/s */
    float* cos_h;    /* written: cos(psi) */
    float* sin_h;    /* written: sin(psi) */
    const float* length; /* wheelbase is 0.6 * length */
} pictura_agent_state;

/* Traffic lights (paper Sec. 3.2, rendering features: disks visible only
 * within a limited angular range, drawn for the approach they govern and
 * culled once the camera faces away).  Device memory, caller-owned, structure
 * of arrays; light l of world w has index w * lights_per_world + l.  A light
 * is a disk of radius `radius` centred at (x, y, z) whose normal is the
 * horizontal unit vector (cos_f, sin_f).  Rule R10: with d = C - centre (C
 * the camera centre of rule R1), h = cos_f * d.x + sin_f * d.y and
 * q = (d.x^2 + d.y^2) + d.z^2 (fp32, in this order), a view draws the light
 * iff h > 0 and h * h >= (cos_max * cos_max) * q.  Rule R11: the disk is 12
 * triangles (centre, rim k, rim k+1 mod 12), rim k = centre +
 * radius * (cos 30k deg * u + sin 30k deg * up) with u = (-sin_f, cos_f, 0),
 * up = (0, 0, 1), the cosines and sines rounded to fp32 and each coordinate
 * computed as x - (r cos) * sin_f, y + (r cos) * cos_f, z + r sin.  Its
 * pixels take class cls[l] (e.g. the signal state). */
typedef struct {
    int32_t num_worlds;
    int32_t lights_per_world;
    const float* x;
    const float* y;
    const float* z;
    const float* cos_f;
    const float* sin_f;
    const float* radius;
    const uint8_t* cls;
    float cos_max;   /* cosine of the visibility cone's half-angle, in [0, 1] */
} pictura_lights;

/* Create a context on HIP device `device`.  Returns PICTURA_EDEVICE when no
 * such device exists.  *out is set to NULL on failure. */
pictura_status pictura_create(int32_t device, pictura_ctx* out);

/* Release all device memory owned by the context.  NULL is ignored. */
void pictura_destroy(pictura_ctx ctx);

/* Message of the last error on this context ("" if none).  Owned by ctx. */
const char* pictura_last_error(pictura_ctx ctx);

/* Copy the static scene to device memory owned by the context (replacing any
 * previous scene and invalidating its bins).  Enqueued on `stream`, which the
 * call waits for; where it replaces a scene it first waits for the whole device,
 * as a render on any stream may read that.  The host arrays may be reused as
 * soon as the call returns.
 * Device memory of the scene before and of its bins is used again where the
 * new scene is of like size (a context then keeps at most 1.5 times what its
 * scene needs); otherwise it is freed before any is allocated.
 * EINVAL: null pointers, num_worlds < 1, offsets not non-decreasing, a class
 * ID of 255.  ERANGE: more than 2^31 - 1 triangles.  ENOMEM: allocation. */
pictura_status pictura_scene_upload(pictura_ctx ctx, const pictura_scene* scene, void* stream);

/* Build the uniform grid of every world: square cells of `cell_size_m`
 * metres covering the world's bounds (ceil(extent / cell) cells per axis);
 * each triangle belongs to the cell holding the centre of its xy bounding
 * box (clamped into the grid); each cell records its triangle range and the
 * 3-D bounding box of its triangles.  The library re-lays the triangles out
 * in cell order.  ESTATE: no scene.  EINVAL: cell_size_m not > 0.
 * ERANGE: more than 2^31 - 1 cells.  Enqueued on `stream`, which the call waits
 * for; where it replaces the scene's bins it first waits for the whole device. */
pictura_status pictura_bin_scene(pictura_ctx ctx, float cell_size_m, void* stream);

/* Render all V = num_worlds * agents_per_world * num_cams views (paper
 * Sec. 3.2, Eq. obs_pv), with the traffic lights attached by
 * pictura_set_lights, if any.  View v = (w * agents_per_world + a) * num_cams + k
 * writes out_cls[v][y][x] (uint8 class; 4 = sky for background) and
 * out_depth[v][y][x] (fp32 view-space depth in metres, +inf for background),
 * row-major, y down.  Both outputs are caller-owned device buffers of
 * V * height * width elements.  ESTATE: scene not binned.  EINVAL: null
 * pointers, num_worlds different from the scene's, rig values out of range
 * (num_cams 1..8, width/height 1..4096, fx, fy > 0, 0 < near < far, far/near
 * small enough for the 24-bit depth key).  Asynchronous on `stream`. */
pictura_status pictura_render_views(pictura_ctx ctx, const pictura_agents* agents, const pictura_rig* rig,
                                    uint8_t* out_cls, float* out_depth, void* stream);

/* Render like pictura_render_views and also a shaded colour image (rule R13;
 * the paper's observations are RGB images, Sec. 3.2, rendering features: agents
 * are cuboids coloured per face with depth-aware brightness).  In this mode a
 * box triangle's visibility key carries a shading id, class | (face + 1) << 4
 * with face 0 bottom, 1 top, 2 back, 3 front, 4 right, 5 left (the order of
 * rule R9's triangles, two per face), in place of its class; every other
 * triangle keeps its class.  out_cls receives key & 15.  out_rgb[v][c][y][x]
 * (uint8, planar, c = red, green, blue): with base = palette[class] / 255
 * (class: R G B -- 0 ground 96 112 72, 1 road 72 72 78, 2 marking 232 232 224,
 * 3 vehicle 52 96 220, 4 sky 140 184 232, 5 curb 160 160 152, 6 pedestrian
 * 224 72 64, 7 wall 168 144 120, 8 red light 255 32 24, 9 amber 255 184 0,
 * 10 green 32 224 96, 11..15 128 128 128), factor = 0.45, 1, 0.55, 0.85, 0.7,
 * 0.7 for the faces bottom .. left and 1 for other surfaces, b = 1 - 0.6 *
 * min(z / far, 1) on box faces (z the output depth) and 1 elsewhere:
 * rint(255 * min(base * (factor * b), 1)), fp32 in this order.  One sample
 * per pixel (pictura_render_rgb_aa antialiases).  Device buffers, caller-owned:
 * out_rgb V*3*H*W bytes.  EINVAL as pictura_render_views, a null out_rgb, or a
 * scene class ID above 15 (agent and light classes are taken modulo 16).
 * Asynchronous on `stream`. */
pictura_status pictura_render_rgb(pictura_ctx ctx, const pictura_agents* agents, const pictura_rig* rig,
                                  uint8_t* out_cls, float* out_depth, uint8_t* out_rgb, void* stream);

/* pictura_render_rgb with analytic-coverage antialiasing at one sample per
 * pixel (rule R14; the paper's production renders smooth edges this way so
 * that thin structures such as lane lines stay visible at low resolution,
 * Sec. 3.2, rendering features, and App. on render quality).  out_cls and
 * out_depth are those of pictura_render_views (the pixel centre's surface).
 * A surface is a snapped 4-gon whose two fan pieces are both drawn and whose
 * turns all have one sign, none zero: a pair of scene triangles (a, b, c),
 * (a, c, d) of one class (see pictura_scene_upload) with all four vertices in
 * front of the near plane and neither triangle wholly beyond far, or a
 * triangle that the near clip turns into a 4-gon; otherwise each fan piece of
 * rule R6 is a surface of its own.  A surface leaves a fragment on every pixel
 * whose centre is within one pixel of its snapped bounding box and that it
 * covers in part: with E_k the edge function of R6 at the centre (no top-left
 * bias) and L_k the edge's length, both in subpixels, c_k = min(max(
 * fma(fl(E_k), fl(1 / (256 L_k)), 0.5), 0), 1), coverage a = min(max(((c_0 +
 * c_1) + c_2) - 2, 0), 1) for a triangle (edges v1->v2, v2->v0, v0->v1) and
 * min(max((((c_0 + c_1) + c_2) + c_3) - 3, 0), 1) for a 4-gon in positive
 * order (edges p_k->p_k+1), a8 = rint(255 a), fp32; the fragment exists when
 * 0 < a8 < 255 and the depth plane of the surface's first piece passes R7's
 * test at the centre.  A pixel keeps its nearest fragment, ordered by o =
 * (key >> 16) << 16 | (key & 255) << 8 | (255 - a8) with key the fragment's R7
 * key.  With key_c the pixel's final key, when o >> 16 <= key_c >> 16 (the
 * fragment is not behind the centre's surface) and (o >> 8) & 255 != key_c &
 * 255 (another shading id), the pixel's colour is (C_o * a8 + C_c * (255 -
 * a8) + 127) / 255 per channel in integers, C_o the R13 colour of the key
 * ((o >> 16) << 16) | ((o >> 8) & 255) and C_c that of key_c; otherwise C_c.
 * During the call the kernel keeps each pixel's nearest fragment in the words
 * of out_depth and writes the depths over them at the end, so out_depth must
 * not overlap out_cls or out_rgb.  Buffers, errors and ordering as
 * pictura_render_rgb. */
pictura_status pictura_render_rgb_aa(pictura_ctx ctx, const pictura_agents* agents, const pictura_rig* rig,
                                     uint8_t* out_cls, float* out_depth, uint8_t* out_rgb, void* stream);

/* Render like pictura_render_views (same out_cls, out_depth) and also the
 * instance visibility the paper's analysis reads from its renderer, each road
 * user's occlusion percentage (Sec. 5.2, "Grounding in What the Cameras
 * See": probes of the trained policy):
 *  - out_inst[v][y][x] (int32): the agent index a (0 .. agents_per_world - 1,
 *    within the view's world) whose box owns the pixel's visible surface: among
 *    the boxes with a fragment whose visibility key (rule R7) equals the pixel's
 *    final key, the lowest index; -1 where no box does (map geometry, traffic
 *    lights, sky).
 *  - out_counts[v][a][2] (uint32): footprint, the pixels agent a's box covers in
 *    view v when drawn alone (rules R2-R7, far plane included), and visible, the
 *    pixels of out_inst equal to a.  The ego's own entry is 0.  Occlusion
 *    fraction = 1 - visible / footprint.
 * Device buffers, caller-owned: out_inst V*H*W int32, out_counts
 * V*agents_per_world*2 uint32 (the library clears it on `stream` first).
 * After the class/depth pass the kernel draws the visible boxes in ascending
 * agent order; a pixel is claimed through one bit in the framebuffer's
 * padding and its owner stored straight into out_inst.  Errors as
 * pictura_render_views, and EINVAL for a null out_inst or out_counts.
 * Asynchronous on `stream`. */
pictura_status pictura_render_instances(pictura_ctx ctx, const pictura_agents* agents, const pictura_rig* rig,
                                        uint8_t* out_cls, float* out_depth, int32_t* out_inst,
                                        uint32_t* out_counts, void* stream);

/* Attach traffic lights (see pictura_lights) to the context: later
 * pictura_render_views calls draw them.  The context keeps the pointers, not
 * a copy: the arrays must stay valid while it renders, and their contents
 * may change between render calls (a signal changing state is a new cls
 * value, ordered on the render stream like any other input).  NULL, or
 * lights_per_world == 0, detaches.  EINVAL: num_worlds < 1, null arrays,
 * lights_per_world > 2^20, cos_max outside [0, 1]; a render call returns
 * EINVAL when num_worlds differs from its scene's.  ERANGE: more than
 * 2^31 - 1 lights.  No device work; synchronous. */
pictura_status pictura_set_lights(pictura_ctx ctx, const pictura_lights* lights);

/* One kinematic-bicycle step for every agent (the per-step agent motion of
 * the headline workload; the paper's simulation step is dt = 0.1 s, App. A.3,
 * Tab. hparams, and its agents follow a kinematic model whose exact form it
 * does not print, so the semi-implicit bicycle below is this library's
 * reading): v' = clamp(v + accel * dt, 0, vmax);
 * psi' = psi + v' / (0.6 length) * tan(steer) * dt wrapped into (-pi, pi];
 * x += v' cos(psi') dt; y += v' sin(psi') dt; cos_h/sin_h = cos/sin(psi').
 * steer[count] (radians) and accel[count] (m/s^2) are device arrays.
 * EINVAL: null pointers, count < 0, dt or vmax not finite.  Asynchronous. */
pictura_status pictura_agents_step(pictura_ctx ctx, const pictura_agent_state* state, const float* steer,
                                   const float* accel, float dt, float vmax, void* stream);

/* ---- introspection and test controls -------------------------------------- */

/* Reference for the achievable HBM write rate (the render's roofline is an
 * HBM write bound): writes `bytes` zero bytes to the device buffer dst with
 * 16-byte non-temporal stores, the store pattern of the render's write-out,
 * and nothing else.  dst must be 16-byte aligned and bytes a multiple of 16
 * (EINVAL otherwise); dst must hold at least `bytes` bytes.  Asynchronous on
 * `stream`: time it with events on that stream. */
pictura_status pictura_store_probe(pictura_ctx ctx, void* dst, uint64_t bytes, void* stream);

/* Grid geometry after pictura_bin_scene (host memory, synchronous: waits for
 * the binning to finish).  dims[w] = nx, ny; cell_base[w] = first cell of
 * world w (cell_base[num_worlds] = total cells); *total_prims = the number of
 * binned primitives.  A primitive is one input triangle, or a pair: input
 * triangles t and t + 1 of one world with the same class where t + 1 is
 * (a, c, d) for t = (a, b, c), bit for bit (a quad split along its diagonal),
 * paired greedily in input order.  The kernels cull and set up a pair once;
 * its two triangles are still drawn by the rules above, each with its own
 * depth plane.  Any pointer may be NULL. */
pictura_status pictura_bins_info(pictura_ctx ctx, int32_t* dims, int64_t* cell_base, int64_t* total_cells,
                                 int64_t* total_prims);

/* Copy the bins to host memory (synchronous).  cell_start[total_cells + 1]:
 * first re-laid-out primitive of each cell; cell_aabb[total_cells][6]: xmin
 * ymin zmin xmax ymax zmax of the cell's primitives (+inf/-inf when empty);
 * perm[total_prims]: for each re-laid-out primitive, the input index of its
 * first triangle, with bit 31 set for a pair. */
pictura_status pictura_bins_copy(pictura_ctx ctx, uint32_t* cell_start, float* cell_aabb, uint32_t* perm);

#define PICTURA_OPT_CULL   1 /* 1 (default): cell + triangle frustum culling; 0: every triangle of the world */
#define PICTURA_OPT_TILE   2 /* 0 (default): the library's choice (64x64 at most, wider or taller where that pays, narrower in small launches); n in 8..64: force n x n tiles (the last row and column ragged) */
#define PICTURA_OPT_STATS  3 /* 1: count the render kernel's work (cells, triangles, pixels); 0 (default): off */
/* Set a context option.  Images never depend on any option. */
pictura_status pictura_set_option(pictura_ctx ctx, int32_t option, int32_t value);

/* Copy the render kernel's accumulated work counters (PICTURA_OPT_STATS) to
 * host memory (synchronous): out[k], k < n, in this order: view tiles, cells
 * in the gathered rectangles, cells passing the rectangle prefilter, cells
 * passing the frustum test, triangles of those cells, boxes passing, box
 * triangles, first-pass survivors, exact batches, triangles clipped at near,
 * snapped triangles with pixels in the tile, of those rasterized by one lane,
 * pixels those lanes tested, triangles rasterized as records, of those on
 * the fp64 edge path, 8x8 blocks tested, blocks passing, first-pass
 * chunks of 64 candidates, then shader-clock cycles summed over waves spent
 * in:
 * prologue, cell and agent tests, first pass, exact pass (with records),
 * record raster (part of the exact pass), final barrier and write-out; then,
 * for the antialiased colour mode: surfaces whose fragments are evaluated
 * packed over the lanes, the window pixels and 64-pixel steps of those,
 * surfaces swept in 8x8 blocks, blocks swept, fragments written.
 * reset != 0 zeroes the counters. */
pictura_status pictura_stats_copy(pictura_ctx ctx, uint64_t* out, int32_t n, int32_t reset);

#define PICTURA_DEVERR_RING_WAIT 1u /* a raster record reserved in a view's record ring was never published */
/* Device-side errors the render kernels found (the kernels cannot return a
 * status): *out receives the OR of the PICTURA_DEVERR_* bits set by every
 * render call on this context since it was created or last reset; 0 means
 * none.  A set bit means an image may be incomplete (the kernel skipped the
 * work it could not do rather than hang).  Synchronous: waits for all work
 * on the context's device.  reset != 0 clears the word.  EINVAL: null out. */
pictura_status pictura_device_errors(pictura_ctx ctx, uint32_t* out, int32_t reset);

/* Device self-check of the reciprocal the kernels use in place of IEEE
 * division where |argument| lies in [2^-12, 2^20) (hardware reciprocal plus
 * one fused Newton step): *mismatches receives the number of fp32 values x
 * whose bit patterns lie in [lo_bits, lo_bits + count) for which it differs
 * from the correctly rounded 1.0f / x.  Synchronous.  EINVAL: null output or
 * a range reaching past the finite floats of lo_bits' sign. */
pictura_status pictura_selftest_rcp(pictura_ctx ctx, uint32_t lo_bits, uint32_t count, uint64_t* mismatches);

/* pictura_selftest_rcp without any device allocation, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same arguments, checks, result and
 * errors as pictura_selftest_rcp.  Its one piece of scratch, the 64-bit
 * mismatch counter, lives in a fixed 256-byte device array that the library
 * holds on every GPU it runs on until the process ends (its address is taken
 * by pictura_create); the counter does not grow with the range, so no range
 * the self-check accepts exceeds it.  The counter is cleared by a kernel at the
 * start of each call.  All contexts on one GPU share that array: calls that
 * overlap on the same GPU (from several host threads) race and may report
 * each other's counts.  ESTATE: the context's device has no scratch address.
 * Synchronous. */
pictura_status pictura_selftest_rcp_noalloc(pictura_ctx ctx, uint32_t lo_bits, uint32_t count, uint64_t* mismatches);

/* The policy's image encoder on rendered views (inference).  Per view: one
 * plane per class and the inverse depth, five 3x3 convolutions with ReLU
 * (padding 1; 32, 64, 64, 128, 128 channels; strides 2, 2, 1, 2, 1), attention
 * of the camera's queries over the feature map, mean over the queries,
 * projection.  Device pointers to contiguous fp32 arrays in PyTorch's layouts:
 * conv_w[i] [out][in][3][3], queries [cams][16][128], in_proj_w [384][128]
 * (query, key, value), out_proj_w and proj_w [128][128]; conv_b[1..4] 16-byte
 * aligned. */
#define PICTURA_ENCODER_WIDTH 128
#define PICTURA_ENCODER_HEADS 4
#define PICTURA_ENCODER_QUERIES 16
#define PICTURA_ENCODER_MAX_CLASSES 32

typedef struct {
    int32_t cams;          /* view v is camera v % cams; 1..4096 */
    int32_t num_classes;   /* 1..PICTURA_ENCODER_MAX_CLASSES; other class IDs have no plane */
    const float* conv_w[5];
    const float* conv_b[5];
    const float* queries;
    const float* in_proj_w;
    const float* in_proj_b;
    const float* out_proj_w;
    const float* out_proj_b;
    const float* proj_w;
    const float* proj_b;
} pictura_encoder;

/* Bytes of workspace an encode of `views` views of height x width takes (bounded:
 * larger batches are encoded in several parts).  Reads only cams and num_classes. */
pictura_status pictura_encoder_workspace(const pictura_encoder* enc, int64_t views, int32_t height, int32_t width,
                                         uint64_t* bytes);

/* Encode views on `stream` of the current device: cls and depth [views][height]
 * [width] as rendered, out [views][128] fp32.  workspace: device memory, 256-byte
 * aligned, in use until the call's work on the stream is done.  EINVAL: a null or
 * misaligned pointer, sizes out of range, or a workspace too small.  Allocates
 * nothing and does not synchronise, so it can be captured in a graph. */
pictura_status pictura_encode_views(const pictura_encoder* enc, const uint8_t* cls, const float* depth, int64_t views,
                                    int32_t height, int32_t width, void* workspace, uint64_t workspace_bytes,
                                    float* out, void* stream);

/* ---- the policy: acting, learning, stepping the weights ---------------------
 * What follows the encoder in the training process the renderer belongs to
 * (paper Sec. 3.3 and App. A.3: categorical actions, clipped policy optimisation
 * with normalised advantages, AdamW).  Like pictura_encode_views these calls take
 * no context: they run on `stream` of the current device, allocate nothing and
 * do not synchronise, so they can be captured in a graph.  (Replays take the numbers
 * that were captured; an AdamW step's among them is its number, so its bias correction
 * is that of the capture.)  Errors are found on the host before anything is launched. */

#define PICTURA_F32  0
#define PICTURA_BF16 1
#define PICTURA_F16  2

#define PICTURA_MAX_ACTIONS (1 << 20)

/* Logits of a head: row n, one decision, has `actions` values of `dtype` from
 * data + n * stride (in elements; stride >= actions) on.  mask (or NULL): byte
 * mask[n * mask_stride + i] is 0 where action i is not allowed in row n
 * (mask_stride 0: the same for every row); what stands at such a place is not
 * looked at.  A logit of -inf is an action of probability zero as well. */
typedef struct {
    const void* data;
    int32_t dtype;        /* PICTURA_F32, PICTURA_BF16 or PICTURA_F16 */
    int32_t actions;      /* 1..PICTURA_MAX_ACTIONS */
    int64_t rows;         /* 0..2^31 - 1 */
    int64_t stride;
    const uint8_t* mask;
    int64_t mask_stride;
} pictura_logits;

/* How actions are drawn.  A pointer, where not NULL, holds a value for each row
 * in place of the scalar before it.  temperature >= 0 (0: the largest logit; +inf:
 * every allowed action of finite logit weighs the same); top_k <= 0, top_p >= 1 and
 * min_p <= 0 are off, a NaN among top_ps or min_ps too. */
typedef struct {
    float temperature;
    int32_t top_k;
    float top_p;
    float min_p;
    const float* temperatures;
    const int32_t* top_ks;
    const float* top_ps;
    const float* min_ps;
} pictura_sampling;

/* Draw one action per row from the random numbers uniform[rows] in [0, 1).
 * With l the allowed logits of a row, d = (l - max l) / temperature and the
 * weights w = rint(2^31 exp(d)) as whole numbers (fp32 up to the rounding, so
 * that no sum below depends on its order; where l - max l is beyond fp32's range w
 * is 0, at any temperature): order the actions by logit, largest
 * first, equal ones by index.  top_k keeps the first top_k of them; top_p of
 * those the shortest prefix whose weights reach max(1, floor(top_p * their sum));
 * min_p (1 at most) drops what weighs less than min_p * 2^31.  With W the sum that is left
 * and t = floor(u * W) (u and top_p cut to 31 bits), out_action[n] is the first
 * index whose running sum, by index, exceeds t, and out_logp[n] = log(w / W), the
 * logarithm of the probability it was drawn with.  temperature 0 takes the first
 * of the largest logits, with out_logp 0.  A row that allows no action, that holds
 * a NaN or +inf at an allowed place, or whose temperature is negative or NaN gets
 * -1 and NaN.  uniform is taken as 0 below 0 and as the largest number below 1
 * from 1 on. */
pictura_status pictura_sample_actions(const pictura_logits* logits, const pictura_sampling* how, const float* uniform,
                                      int64_t* out_action, float* out_logp, void* stream);

/* The decisions a policy loss is taken over, device arrays of `rows` values
 * (values with `values_stride` elements between them).  weights NULL: all 1.  A row
 * with weight 0 or an action outside 0..actions - 1 (what pictura_sample_actions
 * gives a row without actions) counts nothing: its numbers are not looked at and
 * its gradients are 0. */
typedef struct {
    const float* values;
    int64_t values_stride;
    const int64_t* actions;
    const float* old_logp;       /* log-probability the action was drawn with */
    const float* advantages;
    const float* returns;
    const float* old_values;     /* read where value_clip > 0 */
    const float* weights;
    float temperature;           /* > 0: the one the actions were drawn with */
    float clip;                  /* >= 0 */
    float value_clip;            /* > 0: clipped value loss */
    float value_coef, entropy_coef;
    float denominator;           /* 0: the sum of the weights; else what sums are divided by */
    int32_t normalize;           /* 1: advantages - mean over (standard deviation + 1e-8), weighted, over the rows */
} pictura_policy_batch;

#define PICTURA_POLICY_STATS 6   /* loss, policy loss, value loss, entropy, approximate KL, clipped fraction */

/* Bytes of workspace pictura_policy_loss takes for this many rows. */
pictura_status pictura_policy_loss_workspace(int64_t rows, int32_t actions, uint64_t* bytes);

/* Clipped policy loss and its gradient.  Per row, with p the softmax of the allowed
 * logits over temperature, H = -sum p log p, r = exp(log p[action] - old_logp), A the
 * advantage, v the value, R the return:
 *   policy = -min(r A, clamp(r, 1 - clip, 1 + clip) A)
 *   value  = (v - R)^2 / 2; where value_clip > 0 and |v - old| > value_clip, that of
 *            v clamped to old +- value_clip if it is larger (and then constant)
 *   loss   = policy + value_coef value - entropy_coef H
 * and the means of those over the rows, by weight, are out_stats[0..3]; [4] is the
 * mean of (r - 1) - log r, [5] the weight of rows with r outside 1 +- clip.
 * dlogits (the logits' type, dlogits_stride elements between rows) and dvalues
 * [rows] receive the gradient of the mean loss; it is 0 at actions of probability
 * zero.  If no row counts, or the weights add up to 0 and there is no denominator, all are
 * 0.  Sums are taken in a fixed order.
 * workspace: device memory, 256-byte aligned, in use until the call's work on the
 * stream is done.  dlogits may be the logits' own memory (same stride).  EINVAL: a null or
 * misaligned pointer, a value out of range, or a workspace too small. */
pictura_status pictura_policy_loss(const pictura_logits* logits, const pictura_policy_batch* batch, void* workspace,
                                   uint64_t workspace_bytes, float* out_stats, void* dlogits, int64_t dlogits_stride,
                                   float* dvalues, void* stream);

/* Pairs of sequences of decisions, device arrays.  Sequence s is rows offsets[s] to
 * offsets[s + 1] - 1 of the logits; of pair p sequence 2p is preferred to sequence 2p + 1.
 * offsets do not decrease and lie within 0..rows (they are cut to that; a sequence may be
 * empty).  Rows whose action is outside 0..actions - 1 (padding, or what
 * pictura_sample_actions gives a row without actions), rows that allow nothing and rows
 * outside all sequences count nothing: their gradient is 0. */
typedef struct {
    const int64_t* actions;      /* [rows] */
    const int64_t* offsets;      /* [2 pairs + 1] */
    const float* ref_logp;       /* [rows], log-probabilities by the reference policy; NULL: 0 */
    const float* weights;        /* [pairs]; NULL: all 1.  A pair of weight 0 is not looked at */
    int64_t pairs;               /* 0..2^23 */
    float beta;                  /* > 0 */
    float smoothing;             /* 0 or more, below 1: how likely a pair stands the other way round */
    float denominator;           /* 0: the sum of the weights; else what sums are divided by */
    int32_t average;             /* 1: mean over a sequence's rows that count, 0: sum */
} pictura_preferences;

#define PICTURA_PREFERENCE_STATS 4   /* loss, reward of the preferred, of the others, how often it is larger */

/* Bytes of workspace pictura_preference_loss takes. */
pictura_status pictura_preference_loss_workspace(int64_t rows, int32_t actions, int64_t pairs, uint64_t* bytes);

/* Preference loss by paired log ratios, and its gradient.  With l the logarithm of the
 * softmax of the allowed logits at a row's action, D_s = sum (or mean) of l - ref_logp over
 * the rows of sequence s, m = beta (D_2p - D_2p+1),
 *   loss = -(1 - smoothing) log sigmoid(m) - smoothing log sigmoid(-m),
 * and out_stats holds the means by weight over the pairs of the loss, of beta D_2p, of
 * beta D_2p+1 and of m > 0; out_ratios [2 pairs] the D_s.  dlogits (the logits' type,
 * dlogits_stride elements between rows, apart from the logits) receives the gradient of the
 * mean loss; it is 0 at actions of probability zero.  Sums over rows and pairs are taken in
 * fp64 in a fixed order.  If the weights add up to 0 and there is no denominator, the
 * statistics and the gradient are 0.  A NaN or +inf at an allowed place makes its pair NaN.
 * Meant for sequences of like lengths: with heads of up to 64 actions and 1,024 rows a pair or
 * fewer on average, a workgroup takes all rows of a pair, and the call some 10 ns (heads of 12) to
 * 64 ns (of 64) for each row of its longest pair.
 * workspace: device memory, 256-byte aligned, in use until the call's work on the stream is
 * done.  EINVAL: a null or misaligned pointer, a value out of range, or a workspace too
 * small. */
pictura_status pictura_preference_loss(const pictura_logits* logits, const pictura_preferences* pairs, void* workspace,
                                       uint64_t workspace_bytes, float* out_stats, float* out_ratios, void* dlogits,
                                       int64_t dlogits_stride, void* stream);

#define PICTURA_ADAMW_BLOCK 256   /* elements that share a scale of an 8-bit moment */

/* One tensor of an optimizer step: n elements each, contiguous.  With 32 bits
 * the moments are fp32 and the scales NULL.  With 8 bits exp_avg holds int8 codes
 * c in -127..127 and exp_avg_sq uint8 codes, with one fp32 scale s for each block
 * of PICTURA_ADAMW_BLOCK elements (the last one may be shorter): they stand for
 * c |c| / 127^2 * s and (c / 255)^4 * s. */
typedef struct {
    void* param;
    const void* grad;
    void* exp_avg;
    void* exp_avg_sq;
    float* exp_avg_scale;
    float* exp_avg_sq_scale;
    int64_t n;
    int32_t param_dtype;   /* PICTURA_F32, PICTURA_BF16 or PICTURA_F16 */
    int32_t grad_dtype;
} pictura_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;             /* this step's number, from 1 on */
    int32_t bits;             /* of the moments: 32 or 8 */
    const float* grad_factor; /* device: what gradients are multiplied by first, or NULL */
} pictura_adamw;

/* Bytes of workspace pictura_grad_norm takes for these tensors (reads n alone). */
pictura_status pictura_grad_norm_workspace(const pictura_adamw_tensor* tensors, int32_t count, uint64_t* bytes);

/* Norm of all gradients together: out[0] = sqrt(sum g^2), out[1] = min(1, max_norm /
 * (out[0] + 1e-6)), the factor that clips them (a NaN norm gives NaN).  Squares are
 * summed in fp64, in a fixed order.  out: two floats on the device. */
pictura_status pictura_grad_norm(const pictura_adamw_tensor* tensors, int32_t count, float max_norm, void* workspace,
                                 uint64_t workspace_bytes, float* out, void* stream);

/* One AdamW step (weight decay apart from the gradient) of `count` tensors, fp32
 * without contraction: g = grad * grad_factor, m = beta1 m + (1 - beta1) g,
 * v = beta2 v + ((1 - beta2) g) g, param = param (1 - lr weight_decay)
 * - lr / (1 - beta1^step) (m / (sqrt(v) / sqrt(1 - beta2^step) + eps)), rounded once to
 * the parameter's type.  The factors are taken in fp64 and rounded.  With 8 bits
 * the update uses m and v before they are cut: a block's scale is its largest
 * magnitude (0 if that is below 2^-90), m's code the sign and rint(127 sqrt(|m| / s)),
 * v's rint(255 (v / s)^(1/4)), at least 1 where v > 0.  A NaN makes its block's scale
 * NaN.  With 8 bits and eps from 2^-40 on, the update's root and quotient are off by up to
 * a unit of fp32 each.  A block's second moments below 2^-90 count as zero in the next
 * step, where its first ones may not: gradients below 2^-40 take an eps above them.
 * EINVAL: a null pointer where n > 0, a pointer not aligned to its elements,
 * n < 0, step < 1, betas outside [0, 1), or bits other than 32 and 8. */
pictura_status pictura_adamw_step(const pictura_adamw* how, const pictura_adamw_tensor* tensors, int32_t count,
                                  void* stream);

/* What 8-bit moments stand for, in fp32: param and grad are not read; exp_avg_out[k]
 * and exp_avg_sq_out[k] (host arrays of device pointers) receive tensor k's n values. */
pictura_status pictura_adamw_moments(const pictura_adamw_tensor* tensors, int32_t count, float* const* exp_avg_out,
                                     float* const* exp_avg_sq_out, void* stream);

/* ---- a memory over the steps of an episode ----------------------------------
 * Layers for a policy that decides from what it saw before: a gated linear
 * recurrence over sequences of steps, and the norm between such layers.  As the
 * policy's calls above: no context, `stream` of the current device, no allocation,
 * no synchronisation, errors found on the host before anything is launched. */

#define PICTURA_SCAN_STEPS 16   /* steps between the states that a scan saves for its gradient */

/* `batch` sequences of `steps` steps of `channels` channels.  Element (b, t, c) of gates
 * is at gates[b * gates_batch + t * gates_step + c] (strides in elements, 0 or more),
 * likewise inputs (both of `dtype`), and resets[b * resets_batch + t * resets_step],
 * which is not 0 where step t begins anew: what sequence b remembers is forgotten
 * before that step, a NaN too.  Sequences packed one behind the other are one sequence
 * with resets.  state (or NULL: zeros): fp32 [batch][channels], what is remembered
 * before the first step.  batch * channels < 2^31, steps < 2^31. */
typedef struct {
    const void* gates;
    const void* inputs;
    const float* state;
    const uint8_t* resets;   /* or NULL: none */
    int64_t gates_batch, gates_step;
    int64_t inputs_batch, inputs_step;
    int64_t resets_batch, resets_step;
    int64_t batch, steps;
    int32_t channels;        /* 1 or more */
    int32_t dtype;           /* PICTURA_F32, PICTURA_BF16 or PICTURA_F16 */
} pictura_sequences;

/* Bytes of workspace that a scan of these sizes and its gradient take (reads batch,
 * steps, channels and dtype alone). */
pictura_status pictura_gated_scan_workspace(const pictura_sequences* sequences, uint64_t* bytes);

/* Gated linear recurrence over whole sequences: with a = sigmoid(gates),
 *   h_t = a_t h_(t-1) + (1 - a_t) inputs_t,
 * h_(t-1) = 0 where step t is reset, in fp32 (a and 1 - a each to 10 units of 2^-24 of their
 * own, with gates of 16 bits to 10 + 1.3 |gate|; 0 below 2^-126, from gates of 88 on).  An
 * infinite state stays infinite until a reset; a step whose a is 0 makes it a NaN, or, where the
 * steps are cut into tiles, only within its tile.  out (same type, strides of its own, no two
 * elements at one place) receives h_t;
 * last_state (or NULL) fp32 [batch][channels] the state after the last step; saved (or
 * NULL), fp32 [ceil(steps / PICTURA_SCAN_STEPS)][batch][channels], what the gradient
 * needs: the states before steps 0, 16, 32, ...  The same call gives the same bits; where few
 * channels stand against many steps the steps are cut into tiles, which rounds states in
 * another order.  last_state must not overlap state, nor out the inputs.  Of no steps
 * last_state is state (or zeros).  A tile waits for those before it, which have started before
 * it; should the device not run them for a second, the states behind are NaN up to a reset.
 * workspace: device memory, 256-byte aligned, in use until the call's work on the stream
 * is done.  EINVAL: a null or misaligned pointer, sizes or strides out of range, or a
 * workspace too small. */
pictura_status pictura_gated_scan(const pictura_sequences* sequences, void* out, int64_t out_batch, int64_t out_step,
                                  float* last_state, float* saved, void* workspace, uint64_t workspace_bytes, void* stream);

/* Gradient of pictura_gated_scan: from dout (of out; strides 0 or more) and dlast (of
 * last_state; NULL: zeros), with the `saved` of that call (`state` is not read again)
 *   G_t = dout_t + c_(t+1), c_(steps) = dlast, c_t = a_t G_t (0 where step t is reset),
 *   dinputs_t = (1 - a_t) G_t, dgates_t = a_t (1 - a_t) (h_(t-1) - inputs_t) G_t,
 * and dstate (or NULL) = c_0.  Each is rounded to its type once.  dgates and dinputs must
 * not overlap what is read, nor each other.  Errors and workspace as pictura_gated_scan. */
pictura_status pictura_gated_scan_gradient(const pictura_sequences* sequences, const float* saved, const void* dout,
                                           int64_t dout_batch, int64_t dout_step, const float* dlast, void* dgates,
                                           int64_t dgates_batch, int64_t dgates_step, void* dinputs, int64_t dinputs_batch,
                                           int64_t dinputs_step, float* dstate, void* workspace, uint64_t workspace_bytes,
                                           void* stream);

/* One step of the recurrence (steps is 1, sequences->state not read): state fp32
 * [batch][channels] is replaced by h, out[b * out_batch + c] receives it in the inputs'
 * type.  out and the state may each be the inputs' or the gates' own rows (same type, address
 * and stride), and out the state's; any other memory that is written and also read is EINVAL. */
pictura_status pictura_gated_step(const pictura_sequences* sequences, void* out, int64_t out_batch, float* state, void* stream);

#define PICTURA_MAX_NORM (1 << 16)   /* most elements of a normed row */

/* Kinds of 8-bit codes. */
#define PICTURA_INT8 0   /* two's complement, -127..127 */
#define PICTURA_E4M3 1   /* sign, 4 bits of exponent, 3 of mantissa, no infinities, 448 at most (OCP e4m3fn) */

/* Rows to be normed: row n has `width` values of `dtype` from x + n * x_stride on (in
 * elements; 0: the same row for all), and from residual + n * residual_stride where
 * that is not NULL.  weight: [width] of weight_dtype, `dtype` or PICTURA_F32. */
typedef struct {
    const void* x;
    const void* residual;
    const void* weight;
    int64_t x_stride, residual_stride;
    int64_t rows;          /* 0..2^31 - 1 */
    int32_t width;         /* 1..PICTURA_MAX_NORM */
    int32_t dtype;         /* PICTURA_F32, PICTURA_BF16 or PICTURA_F16 */
    int32_t weight_dtype;
    float eps;             /* 0 or more, finite */
} pictura_norm;

/* Root-mean-square norm with the residual's addition: s = x + residual, rounded to dtype,
 * q = 1 / sqrt(mean(s^2) + eps), out = (s q) weight, rounded to dtype once.  The mean is
 * taken in fp64 and q rounded to fp32.  sum (or NULL) receives s and may be x's or
 * residual's own memory (same stride), as may out; factors (or NULL), fp32 [rows], receives
 * q.  EINVAL: a null or misaligned pointer, or a value out of range. */
pictura_status pictura_rms_norm(const pictura_norm* norm, void* sum, int64_t sum_stride, void* out, int64_t out_stride,
                                float* factors, void* stream);

/* The norm with an output in 8 bits: with y = (s q) weight in fp32, M the largest |y| of the
 * row and L the kind's largest value (127 or 448), scales[n] = M / L and the codes are
 * y (L (1 / M)), every operation rounded to fp32, then to the nearest of the kind, ties to
 * even: they stand for code * scales[n].  A row whose M is below 2^-100 gets scale 0 and codes 0; an infinity or a NaN
 * makes the values of its row NaN.  codes: one byte each, rows codes_stride apart. */
pictura_status pictura_rms_norm_codes(const pictura_norm* norm, int32_t kind, void* sum, int64_t sum_stride, void* codes,
                                      int64_t codes_stride, float* scales, void* stream);

/* What codes stand for, in fp32: out[n * out_stride + i] = code * scales[n].  EINVAL also where
 * out overlaps the codes or the scales. */
pictura_status pictura_row_values(const void* codes, int64_t codes_stride, const float* scales, int32_t kind, int64_t rows,
                                  int32_t width, float* out, int64_t out_stride, void* stream);

/* Bytes of workspace that the gradient takes (reads rows, width and the types alone). */
pictura_status pictura_rms_norm_gradient_workspace(const pictura_norm* norm, uint64_t* bytes);

/* Gradient of pictura_rms_norm: norm->x is its sum (what it normed), residual NULL, factors
 * its factors; from dout (of out) and dsum (of sum; or NULL: zeros), with k = dout weight
 * and u = x q, dx = q (k - u mean(k u)) + dsum, the gradient of x and of the residual
 * alike, rounded to dtype once, and dweight = sum over the rows of dout u, in the weight's
 * type, summed in a fixed order (a workgroup's rows in fp32, the
 * workgroups in fp64).  dx may be dout's or dsum's own memory (same stride).
 * With no rows dweight is 0.  Errors as pictura_rms_norm; workspace: device memory,
 * 256-byte aligned, in use until the call's work on the stream is done. */
pictura_status pictura_rms_norm_gradient(const pictura_norm* norm, const float* factors, const void* dout, int64_t dout_stride,
                                         const void* dsum, int64_t dsum_stride, void* dx, int64_t dx_stride, void* dweight,
                                         void* workspace, uint64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PICTURA_H */
